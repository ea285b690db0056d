"""A layer's code scratch: what a captured call refers to stays where it is when a later call needs more."""
import pytest
import torch

from paper_2507_14811_b200.layer import SegQuantLinear


def bare_layer(K, dual):
    layer = object.__new__(SegQuantLinear)                   # the buffers alone: no weights, no GPU
    layer.device, layer.K, layer.dual = torch.device("cpu"), K, dual
    layer._scratch, layer._outgrown = None, []
    return layer


def test_a_buffer_that_was_handed_out_stays():
    """A CUDA graph holds the address that it was captured with; freeing the buffer under it would let its replays write into
    whatever is put there next."""
    layer = bare_layer(256, True)
    first = layer.scratch_for(10)
    address = first.data_ptr()
    first.fill_(7)
    del first
    later = [layer.scratch_for(M) for M in (100, 1000, 30)]
    assert all(t.numel() >= n for t, n in zip(later, (100 * 512, 1000 * 512, 30 * 512)))
    assert later[1].data_ptr() == later[2].data_ptr()        # no new one for fewer rows
    kept = [t for t in layer._outgrown if t.data_ptr() == address]
    assert len(kept) == 1 and bool(torch.all(kept[0] == 7))


def test_growth_is_bounded():
    """Calls of ever more rows: what is kept stays within the size of the largest buffer, and buffers are few."""
    layer = bare_layer(128, False)
    for M in range(1, 5000, 7):
        layer.scratch_for(M)
    sizes = [t.numel() for t in layer._outgrown] + [layer._scratch.numel()]
    assert sum(sizes[:-1]) <= sizes[-1] and len(sizes) <= 16


@pytest.mark.gpu
def test_a_captured_block_behind_a_larger_call():
    """The replay writes its codes where they were when it was captured, and nowhere into tensors made since."""
    g = torch.Generator().manual_seed(1)
    fc = SegQuantLinear(torch.randn((256, 384), generator=g) * 0.05, None, [0, 384], [0, 256], True)
    fc.calibrate(torch.randn((64, 384), generator=g).to(torch.bfloat16))
    R = torch.randn((700, 384), generator=g).to("cuda").to(torch.bfloat16)
    fc.forward_block(R)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, Y = fc.forward_block(R)
    fc.forward_block(torch.zeros((5000, 384), dtype=torch.bfloat16, device="cuda"))
    others = [torch.full((n,), 9, dtype=torch.uint8, device="cuda") for n in (1 << 16, 1 << 18, 1 << 19, 1 << 20) for _ in range(8)]
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(Y, fc.forward_block(R)[1])
    assert all(bool(torch.all(t == 9)) for t in others)
