"""Bounds of blocks (ipot_enable_blocks) after captured calls that are replayed over other rows: they are those of the rows that are there, as after the calls themselves."""
import pytest
import torch

from paper_2410_01518_b200 import ipot
from parity import make_pot
from test_blocks_gpu import DT, attend, check_bounds, config, pot_rows, verify


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("deferred", [False, True])
@pytest.mark.parametrize("first,n,R", [(10, 5, 16), (10, 1, 16), (37, 100, 32), (16, 3, 16), (0, 7, 64), (127, 1, 128)])
def test_a_replayed_append_of_other_rows(first, n, R, deferred, dtype):
    """Rows of larger values first, then of smaller ones: the second replay's bounds lie within the first's."""
    cfg = config(dtype, 2, 1, 4, 2, 64, 200)
    g = torch.Generator(device="cuda").manual_seed(first + n)
    make = lambda m, size: size * torch.randn((2, 1, 2, m, 64), generator=g, device="cuda").to(DT[dtype])  # noqa: E731
    h = make_pot(cfg)
    s = torch.cuda.Stream()
    try:
        torch.cuda.synchronize()
        ipot.ipot_set_stream(h, s.cuda_stream)
        ipot.ipot_enable_blocks(h, R)
        if first:
            K0, V0 = make(first, 0.5), make(first, 1.0)
            ipot.ipot_append_chunk(h, K0, V0, first)
        K, V = make(n, 4.0), make(n, 1.0)
        torch.cuda.synchronize()
        if deferred:
            ipot.ipot_set_deferred_append(h, True)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=s):
            ipot.ipot_set_stream(h, s.cuda_stream)
            ipot.ipot_append_chunk(h, K, V, n)
            ipot.ipot_view(h)   # (a deferred append's rows are copied by the call that needs them)
        for size in (4.0, 0.25, 2.0, 0.125):
            K.copy_(make(n, size))
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                gr.replay()
            s.synchronize()
            keys, values = pot_rows(h, cfg, first + n)
            assert torch.equal(keys[:, :, :, first:], K)
            check_bounds(h, cfg, keys, R)
        q = torch.randn((2, 1, 4, 64), generator=g, device="cuda").to(DT[dtype])
        torch.cuda.synchronize()
        blocks = min(2, -(-(first + n) // R))
        verify(cfg, q, keys, values, R, blocks, *attend(h, cfg, q, blocks))
        del gr
    finally:
        torch.cuda.synchronize()
        ipot.ipot_destroy(h)
