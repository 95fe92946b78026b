"""Sizes of the 4-bit head's calls that the host refuses or takes, without a GPU: every call here ends at a check of its arguments."""
import ctypes

import pytest

import paper_2411_18462_amd as svip

SHAPE, ALIGN = 2, 4


@pytest.mark.parametrize("rows,runs,fp32,others", [(3728270, 36, ALIGN, ALIGN), (384578, 349, SHAPE, ALIGN), (262657, 511, SHAPE, ALIGN), (1 << 18, 512, SHAPE, SHAPE)])
def test_runs_of_quantize_mx(rows, runs, fp32, others):
    """Of runs of 128 columns, here 2^27 - 8, - 6, - 1 and 2^27, fewer than 2^27, and in fp32, with 32 lanes to a run, at most 2^27 - 8: whole workgroups of more would
    be 2^32 threads, which no launch takes.  Codes that are not on 16 bytes end a call behind the check of its sizes."""
    lib = svip.load()
    buf = ctypes.create_string_buffer(1 << 12)
    p = (ctypes.addressof(buf) + 255) & ~255                     # a fake, aligned "device" pointer, never dereferenced
    call = lambda dtype: lib.svip_quantize_mx(p, dtype, rows, 128 * runs, 128 * runs, p + 8, 64 * runs, p, 4 * runs, None)  # noqa: E731
    assert call(0) == fp32 and call(1) == call(2) == others


def test_workspace_of_the_sampler():
    """What svip.h says of its size."""
    import torch

    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for N, V in ((1, 1), (1, 4096), (1, 4097), (7, 9000), (1088, 151936), (1 << 20, 8), (3, 1 << 22)):
            need = N * (64 + 4896 * -(-V // 4096))
            assert svip.sample_workspace_bytes(dtype, N, V) == 512 + -(-need // 256) * 256
