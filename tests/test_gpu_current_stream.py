"""The handle of the current stream that the binding gives to the library is the one that torch documents."""
import pytest
import torch

from paper_2605_18071_amd import kvd

pytestmark = pytest.mark.gpu


def test_the_handle_is_that_of_the_current_stream():
    here = torch.cuda.current_device()
    assert kvd._raw_stream(here) == torch.cuda.current_stream(here).cuda_stream == torch.cuda.default_stream(here).cuda_stream
    seen = set()
    for stream in (torch.cuda.Stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            assert kvd._raw_stream(here) == torch.cuda.current_stream(here).cuda_stream == stream.cuda_stream
            seen.add(kvd._raw_stream(here))
    assert len(seen) == 2 and kvd._raw_stream(here) not in seen
    graph, x = torch.cuda.CUDAGraph(), torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        assert kvd._raw_stream(here) == torch.cuda.current_stream(here).cuda_stream == stream.cuda_stream
        x += 1
    graph.replay()
    torch.cuda.synchronize()
    assert (x == 1).all()
