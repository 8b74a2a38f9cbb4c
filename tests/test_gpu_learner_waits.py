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
    assert kernels.run_uneven_wait and kernels.run_load_and_end


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


def _load_and_end(kernels, stages, used, arrivals, limit):
    import torch

    data = torch.randint(1, 256, (max(stages, 1) * 1024,), dtype=torch.uint8, device="cuda")
    missing = torch.zeros(1, dtype=torch.int32, device="cuda")
    took = torch.zeros(1, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    assert kernels.run_load_and_end(C.c_void_p(data.data_ptr()), stages, used, arrivals, C.c_longlong(limit), C.c_void_p(missing.data_ptr()),
                                    C.c_void_p(took.data_ptr())) == 0
    return int(missing), int(took)


@pytest.mark.gpu
@pytest.mark.parametrize("stages,used", [(0, 0), (1, 0), (3, 0), (4, 0), (4, 4), (5, 1), (7, 3), (9, 5), (12, 8), (12, 12)])
def test_a_loading_warp_ends_with_its_copies_landed(kernels, stages, used):
    # whoever uses them stops after `used` stages; the loader issues the rest into the free part of the ring
    missing, _ = _load_and_end(kernels, stages, used, 1, 1_000_000_000)
    assert missing == 0


@pytest.mark.gpu
def test_its_end_is_bounded(kernels):
    # barriers that wait for an arrival that never comes: one limit, not one for every stage
    limit = 2_000_000
    _, took = _load_and_end(kernels, 4, 0, 2, limit)
    assert limit < took < 2 * limit


@pytest.mark.gpu
def test_every_stream_is_told_once(kernels):
    import torch

    torch.zeros(1, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    told = [kernels.run_told(count, *[C.c_void_p(s.cuda_stream) for s in streams]) for count in (0, 0, 1, 1, 5, 5)]
    assert told == [0, 0, 7, 0, 7, 0]


@pytest.mark.gpu
def test_sync_waits_for_its_own_stream_only():
    import torch
    from paper_1509_04210_b200 import learner as L

    L.sync()
    side = torch.cuda.Stream()
    done = torch.cuda.Event()
    torch.cuda.synchronize()
    torch.cuda._sleep(1_000_000_000)            # half a second on the legacy stream
    done.record()
    with torch.cuda.stream(side):
        L.sync()
        assert not done.query()
        torch.cuda._sleep(200_000_000)
        own = torch.cuda.Event()
        own.record()
        L.sync()
        assert own.query()
    torch.cuda.synchronize()
