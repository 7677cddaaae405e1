"""The give-up paths of the 16-bit kernels: their waits run on barriers that nobody completes, end within their limit and
leave a status; nothing is filled, and no tensor memory freed, over what was given up on."""
import ctypes
import os
import subprocess
import time

import pytest
import torch

from paper_2609_35800_gb300 import build

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("probe") / "attention_wait_probe.so")
    subprocess.run([build.nvcc()] + build.ARCH + build.NVCC_FLAGS + ["-shared", os.path.join(HERE, "attention_wait_probe.cu"),
                                                                     "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.run_ring.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    lib.run_slow.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int]
    lib.run_products.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int]
    return lib


def test_a_place_is_not_filled_over_a_copy_that_was_given_up_on(probe):
    for _ in range(2):
        status = torch.zeros(4, dtype=torch.int32, device="cuda")
        result = torch.full((5,), 7, dtype=torch.int32, device="cuda")
        assert probe.run_ring(status.data_ptr(), result.data_ptr()) == 0
        torch.cuda.synchronize()
        # nobody's wait was met, nothing was filled again, and everybody left
        assert result.tolist() == [0, 0, 0, 0, 1]
        assert status.tolist() == [1, 0, 0, 0]


def test_a_wait_lasts_about_a_second(probe):
    """Long enough for a copy behind anything that the memory may be busy with, and the end of a launch that is stuck."""
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    result = torch.zeros(5, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    begin = time.perf_counter()
    assert probe.run_ring(status.data_ptr(), result.data_ptr()) == 0
    torch.cuda.synchronize()
    waits = (time.perf_counter() - begin) / 2  # a wait, then a drain
    assert 0.5 <= waits <= 4.0


@pytest.mark.parametrize("moves", [1, 0])
def test_whoever_has_nothing_to_do_waits_as_long_as_others_move(probe, moves):
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    result = torch.full((2,), 7, dtype=torch.int32, device="cuda")
    assert probe.run_slow(status.data_ptr(), result.data_ptr(), 3_000_000_000, moves) == 0
    torch.cuda.synchronize()
    assert result.tolist() == [moves, 1 - moves]
    assert status.tolist() == [1 - moves, 0, 0, 0]


def test_products_have_ended_before_tensor_memory_is_freed(probe):
    for steps in (1, 2000, 8):  # (and a launch after one that gave up has its tensor memory)
        status = torch.zeros(4, dtype=torch.int32, device="cuda")
        result = torch.zeros(3, dtype=torch.int32, device="cuda")
        assert probe.run_products(status.data_ptr(), result.data_ptr(), steps) == 0
        torch.cuda.synchronize()
        assert result.tolist() == [0, 1, 128 * 128]
        assert status.tolist() == [1, 0, 0, 0]
