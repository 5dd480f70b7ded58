"""The operators' waits on the GPU are bounded: one that nothing ends gives up after about two seconds,
with one answer for its warp, and ends the block's other waits."""
import ctypes as C
import os
import subprocess

import pytest

pytest.importorskip("torch")

from paper_2608_15762_gb300 import build  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "wait_check.cu")
    so = str(tmp_path_factory.mktemp("waits") / "wait_check.so")
    subprocess.check_call([build.nvcc()] + build.ARCH + build.FLAGS + ["-shared", "-o", so, src])

    def run(which):
        out = (C.c_int * 196)()
        assert C.CDLL(so).wait_check(which, out) == 0
        return list(out)
    return run


def test_a_wait_that_gives_up_has_one_answer_for_its_warp(check):
    v = check(0)
    assert v[:32] == [0] * 32 and v[32:64] == [1] * 32      # half of warp 0's lanes had their phase
    assert v[64:128] == [1] * 64
    assert v[128:192] == [0] * 64
    assert v[192:194] == [1, 1]
    assert 1900 <= v[194] <= 4000 and v[195] < 1000


def test_warps_that_meet_see_what_the_others_wrote_and_wait_no_longer_than_others(check):
    v = check(1)
    assert v[0] == 0 and v[1] == 1
    assert 1900 <= v[2] <= 4000 and v[3] < 1000
