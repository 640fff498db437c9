"""A selection on another stream than the one on which its holder was made."""
import pytest
import torch

from test_gpu_beams import DEV, check, make, random_inputs

pytestmark = pytest.mark.gpu


def test_a_holder_is_ready_for_any_stream():
    logits, scores = random_inputs(3, 4, 5000, torch.float16)
    want = check(make(3, 4, 5000), logits, scores)
    nbytes = make(3, 4, 5000).workspace.numel()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        old = torch.full((nbytes,), 7, dtype=torch.uint8, device=DEV)    # what the allocator hands out next
        del old
        torch.cuda._sleep(20_000_000)                     # some 10 ms of work before what the holder clears
        sel = make(3, 4, 5000)
        got = [sel.select(logits, scores, stream=side) for _ in range(2)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
