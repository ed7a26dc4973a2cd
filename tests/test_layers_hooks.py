"""The layers' testing hooks and choice of kernels, on the host."""
import ctypes as C

import torch

from paper_2401_14110_b200 import binding as lba


def test_wait_override_numbers():
    lib = lba.load_library()
    assert lib.lba_set_wait_override(4) == -2 and lib.lba_set_wait_override(-1) == -2
    assert lib.lba_set_wait_override(1) == 0 and lib.lba_set_wait_override(0) == 0


def test_few_rows_take_the_faster_side():
    # the kernel for few rows needs no workspace; sizes far on either side of its rule, where it took 0.4 to 0.8 and 1.4 to 2.3 times as long
    size = lambda M, N, K, gated=False: lba.backward_workspace_bytes(M, N, K, 1, N, torch.bfloat16, activation="silu", gated=gated)  # noqa: E731
    assert not any(size(*s) for s in [(1, 512, 512), (4, 8192, 8192), (17, 4096, 4096), (32, 2048, 2048), (48, 4096, 512), (64, 2048, 512)])
    assert all(size(*s) for s in [(64, 2048, 4096), (64, 4096, 4096), (64, 8192, 2048), (64, 8192, 1024, True), (48, 8192, 1024, True), (64, 512, 4096), (65, 512, 512)])


def test_sizes_beyond_the_tensor_copies_are_refused():
    lib = lba.load_library()
    how = lba._Backward()
    how.activation, how.preact = 4, 256
    fake, most = C.c_void_p(256), (1 << 31) - 1
    for M, N, K in [(most, most >> 1, 1), (most, most >> 1, most), (1 << 20, 1 << 18, 1), (1 << 20, 1, 1 << 19), (1, 1 << 19, 1 << 19)]:   # dz: up to 2^64.6 bytes
        assert lib.lba_gated_backward(fake, fake, fake, fake, fake, 1, fake, fake, 1, M, N, K, C.byref(how), fake, fake, fake, fake, fake, fake,
                                      C.c_size_t(1 << 63), None) == -2
        assert lib.lba_backward_workspace_bytes(1, M, N, K, 1, 1, C.byref(how), 7) == 0
    assert lib.lba_backward_workspace_bytes(1, 1 << 20, (1 << 18) - 64, 64, 1, 1, C.byref(how), 7) > 2 << 40   # more than a GPU holds, and all strides in range
