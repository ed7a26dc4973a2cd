"""Calls with an explicit stream while the current stream still has work queued on memory that it has given back.  Needs a B200."""
import pytest
import torch

from paper_2401_14110_b200 import binding as lba
from paper_2401_14110_b200 import code_domain_formats, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PROD, ACC = code_domain_formats(7, 4)
M, N, K = 1024, 1536, 1024
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def operands():
    A, sa = (t.to(DEV) for t in synth.quantise_per_tensor(synth.gaussian((M, K), 1)))
    B, sb = (t.to(DEV) for t in synth.quantise_per_tensor(synth.gaussian((N, K), 2)))
    return A, B, sa, sb, synth.gaussian((M, N), 3).to(BF16).to(DEV), synth.gaussian((2, M, N), 4).to(BF16).to(DEV)


CALLS = {  # what a call allocates in bytes, and the call
    "gemm": ([4 * M * N], lambda A, B, sa, sb, g, z, **kw: [lba.lba_gemm(A, B, sa, sb, None, PROD, ACC, **kw)]),
    "linear": ([2 * M * N, 4 * M * N], lambda A, B, sa, sb, g, z, **kw: lba.lba_linear(A, B, sa, sb, None, PROD, ACC, out_dtype=BF16, preact=torch.float32, **kw)),
    "gated": ([M * N, 4 * M * N], lambda A, B, sa, sb, g, z, **kw: lba.lba_gated(A, B, B, sa, sb, sb, None, None, PROD, ACC, out_dtype=torch.uint8, out_scale=sa, preact=BF16, **kw)),
    "linear_backward": ([lba.backward_workspace_bytes(M, N, K, 1, 1, BF16, "gelu"), 2 * M * K, 2 * N * K],
                        lambda A, B, sa, sb, g, z, **kw: lba.lba_linear_backward(g, A, B, sa, sb, PROD, z[0], "gelu", **kw)),
    "gated_backward": ([lba.backward_workspace_bytes(M, N, K, 1, 1, BF16, "silu", gated=True), 2 * M * K, 2 * N * K],
                       lambda A, B, sa, sb, g, z, **kw: lba.lba_gated_backward(g, A, B, B, sa, sb, sb, PROD, z, **kw)),
}


@pytest.mark.parametrize("by_handle", [False, True])
@pytest.mark.parametrize("name", list(CALLS))
def test_memory_that_is_still_in_use_is_left_alone(name, by_handle, operands):
    sizes, call = CALLS[name]
    side = torch.cuda.Stream()
    want = [t.clone() for t in call(*operands)]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    call(*operands, stream=side)   # (memory of that stream's own)
    torch.cuda.synchronize()
    held = [torch.full((size,), 7, dtype=torch.uint8, device=DEV) for size in sizes]   # what the call would be given first if it took it here
    kept = [torch.empty_like(t) for t in held]
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)   # some 50 ms
    for k, t in zip(kept, held):
        k.copy_(t)
    del t, held
    got = call(*operands, stream=side.cuda_stream if by_handle else side)
    side.synchronize()
    assert not torch.cuda.current_stream().query()   # the copies are still to come
    torch.cuda.synchronize()
    assert all(bool((k == 7).all()) for k in kept)
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_results_given_back_are_not_reused_under_the_current_stream(operands):
    side, other = torch.cuda.Stream(), operands[2] * 2
    torch.cuda.synchronize()
    for _ in range(3):
        got = CALLS["linear_backward"][1](*operands, stream=side)
        side.synchronize()
        torch.cuda._sleep(20_000_000)
        kept = got[1].clone()
        del got
        CALLS["linear_backward"][1](operands[0], operands[1], other, *operands[3:], stream=side)
        want = CALLS["linear_backward"][1](*operands)[1]
        torch.cuda.synchronize()
        assert torch.equal(kept, want)


def test_nan_codes_are_counted_behind_the_count():
    codes = torch.full((1000,), 0x7F, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    assert lba.count_nan_codes(codes, stream=side) == 1000
    assert lba.count_nan_codes(codes) == 1000
