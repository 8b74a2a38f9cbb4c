"""The bounded waits of the product kernels, by themselves and with limits that run out."""
import ctypes as C
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCE = os.path.join(HERE, "kernels", "waits.cu")


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    from paper_1509_04210_b200 import build

    out = str(tmp_path_factory.mktemp("waits") / "waits.so")
    subprocess.check_call([os.environ.get("NVCC", "nvcc")] + build.NVCC_FLAGS + ["-o", out, SOURCE])
    return C.CDLL(out)


def test_the_kernels_of_this_test_build(kernels):
    assert kernels.run_uneven_wait


@pytest.mark.gpu
@pytest.mark.parametrize("low,high,after", [
    (20_000, 30_000, 0),                    # nobody comes
    (50_000, 500_000_000, 1_000_000),       # half of the lanes would give up, the others not
    (500_000_000, 500_000_000, 100_000),    # in time
])
def test_the_lanes_of_a_warp_get_one_answer(kernels, low, high, after):
    import torch

    answers = torch.full((1,), 12345, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    i64 = C.c_longlong
    assert kernels.run_uneven_wait(i64(low), i64(high), i64(after), C.c_void_p(answers.data_ptr())) == 0
    assert int(answers) == (-1 if low > after > 0 else 0)
