"""The operators on token states on the GPU at the edge of what is documented: first calls of several threads, large caps, weights and gradients at
the ends of a type's range, buffers that autograd holds."""
import numpy as np
import pytest
import torch

import encoder_reference as ref
import paper_2210_02574_amd as pkg
import workloads as wl

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def he():
    assert torch.cuda.is_available(), "this test needs the MI355X"
    return pkg.HE.from_params(wl.C1B, device=0)


def rand(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g)).to(dtype).cuda()


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def offsets_of(lengths):
    return i32(*np.concatenate([[0], np.cumsum(lengths)]).tolist())


def test_a_context_knows_its_stream_before_it_says_that_it_is_ready():
    """A second thread that finds the extension in place calls at once: its kernels belong on its own current stream then."""
    streams = []

    class Watched(pkg.HE):
        def __setattr__(self, name, value):
            if name == "_tensors" and value is not None:
                streams.append(self._raw_stream(0))
            super().__setattr__(name, value)

    he, side, x = Watched.from_params(wl.C1B, device=0), torch.cuda.Stream(), rand(1, 3, 8)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        he.pool_mean(x, i32(0, 3))
    torch.cuda.synchronize()
    assert streams == [side.cuda_stream]
