"""Two builds of the library in one process share no state: each counts its own launches."""
import ctypes
import subprocess

import pytest
import torch

from paper_2602_02071_b200 import binding, build


def test_no_symbol_is_unique_to_the_process():
    for lib in (build.build(), build.build_wait_test()):
        names = subprocess.run(["nm", "-D", "--defined-only", lib], check=True, capture_output=True, text=True).stdout.splitlines()
        assert len(names) > 20 and not [n for n in names if n.split()[-2] == "u"]


@pytest.mark.gpu
def test_each_library_counts_its_own_launches():
    other = ctypes.CDLL(build.build_wait_test())
    other.baps_hif8_encode.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    other.baps_launch_count.restype = ctypes.c_int64
    x = torch.randn(4096, device="cuda")
    codes = torch.empty(4096, dtype=torch.uint8, device="cuda")
    want = binding.baps_hif8_encode(x)
    assert other.baps_hif8_encode(x.data_ptr(), codes.data_ptr(), 4096, None) == 0     # (tables are built)
    torch.cuda.synchronize()
    assert torch.equal(codes, want)
    here, there = binding.launch_count(), other.baps_launch_count()
    for _ in range(3):
        assert other.baps_hif8_encode(x.data_ptr(), codes.data_ptr(), 4096, None) == 0
    assert (binding.launch_count(), other.baps_launch_count()) == (here, there + 3)
    binding.baps_hif8_encode(x)
    assert (binding.launch_count(), other.baps_launch_count()) == (here + 1, there + 3)
