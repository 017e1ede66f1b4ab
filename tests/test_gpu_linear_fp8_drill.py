"""A wait of the 8-bit linear layer that runs out comes back as a status, and the kernels work right afterwards."""
import ctypes

import pytest
import torch

from paper_2211_17192_b200 import binding

pytestmark = pytest.mark.gpu


def test_waits_that_run_out_are_reported_and_leave_the_kernels_usable():
    h = binding.lib()
    h.spec_timeout_drill.restype = ctypes.c_int
    h.spec_timeout_drill.argtypes = [ctypes.c_void_p]
    g = torch.Generator(device="cuda").manual_seed(1)
    w = binding.spec_quantize_fp8(torch.randn(700, 1024, device="cuda", generator=g))
    xs = [binding.spec_quantize_fp8(torch.randn(rows, 1024, device="cuda", generator=g)) for rows in (3, 300)]  # (either kernel)
    want = [binding.spec_linear_fp8(*x, *w) for x in xs]
    torch.cuda.synchronize()
    assert binding.spec_device_error() == 0
    for _ in range(3):  # (tensor memory that was not freed would be missing in the next call)
        assert h.spec_timeout_drill(torch.cuda.current_stream().cuda_stream) == -6, h.spec_last_error().decode()
        codes = [int(c) for c in h.spec_last_error().decode().split("codes ")[1].split(")")[0].split(",")]
        assert len(codes) == 4 and 1 <= codes[2] <= 6 and 16 <= codes[3] <= 26
        assert binding.spec_device_error() == 0
        for x, y in zip(xs, want):
            assert torch.equal(binding.spec_linear_fp8(*x, *w), y)
    assert binding.spec_device_error() == 0


def test_a_drill_beside_clusters_of_another_stream():
    # the drills' CTAs and those of the layer's clusters all take tensor memory, and wait for CTAs on other SMs
    h = binding.lib()
    h.spec_timeout_drill.restype = ctypes.c_int
    h.spec_timeout_drill.argtypes = [ctypes.c_void_p]
    g = torch.Generator(device="cuda").manual_seed(2)
    w = binding.spec_quantize_fp8(torch.randn(4096, 4096, device="cuda", generator=g))
    x = binding.spec_quantize_fp8(torch.randn(5, 4096, device="cuda", generator=g))
    want = binding.spec_linear_fp8(*x, *w)
    side, got = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(side):
            got += [binding.spec_linear_fp8(*x, *w) for _ in range(40)]
        assert h.spec_timeout_drill(torch.cuda.current_stream().cuda_stream) == -6, h.spec_last_error().decode()
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in got) and binding.spec_device_error() == 0
