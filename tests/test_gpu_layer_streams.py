"""Weights quantised on a stream of the caller's own: the memory they get is that stream's, not memory that the current stream's queued work still reads."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("kind", ["torch", "raw"])
def test_quantised_weights_do_not_take_what_the_current_stream_still_reads(kind):
    from paper_2508_12801_b200 import binding as ms
    from paper_2508_12801_b200.layer import MoELayer
    E, d, f = 8, 512, 1024
    layer = MoELayer(ms.make_params(16, d, E, 2, io_dtype=ms.BF16), f, training=False, int8=True)
    g = torch.Generator().manual_seed(1)
    w_up, w_down = (torch.randn(E, *s, generator=g).to(torch.bfloat16).to(DEV) for s in ((d, 2 * f), (f, d)))
    want = [t.clone() for pair in layer.quantise(w_up, w_down) for t in pair]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    sizes = [t.numel() * t.element_size() for t in want]
    for _ in range(3):
        # copies that wait on the current stream; their sources go back to its part of the allocator
        old = [torch.full((n,), 77, dtype=torch.uint8, device=DEV) for n in sizes]
        torch.cuda._sleep(100_000_000)                                      # some 50 ms
        copies = [t.clone() for t in old]
        del old
        got = layer.quantise(w_up, w_down, stream=other if kind == "torch" else other.cuda_stream)
        torch.cuda.synchronize()
        assert all((c == 77).all() for c in copies)
        assert all(torch.equal(a, b) for a, b in zip(want, (t for pair in got for t in pair)))
