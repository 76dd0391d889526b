"""A tensor in eight bits without channels is refused like any other wrong one, with a ValueError: on the CPU with stand-ins that
pass for GPU tensors, on the GPU with tensors."""
import pytest

import paper_2208_05419_amd as afno

torch = pytest.importorskip("torch")


class Stand:
    """What the checks look at of a contiguous GPU tensor."""
    is_cuda, device = True, torch.device("cuda", 0)

    def __init__(self, *shape, dtype):
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True


def refused(empty, channels, w, g):
    x = afno.Mx8(*empty, channels)
    for call in (lambda: afno.mx8_unpack(x), lambda: afno.mx8_linear_forward(x, x), lambda: afno.mx8_linear_backward(g, x, w)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("channels", [0, -5])
@pytest.mark.parametrize("rows", [0, 3])
def test_refused(rows, channels):
    e4m3, e8m0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    refused((Stand(rows, 0, dtype=e4m3), Stand(rows, 0, dtype=e8m0)), channels, Stand(0, 7, dtype=torch.bfloat16),
            Stand(rows, 7, dtype=torch.bfloat16))


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [0, 3])
def test_refused_on_the_gpu(rows):
    refused(afno.mx8_empty((rows, 0), "cuda")[:2], 0, torch.empty(0, 7, device="cuda"), torch.zeros(rows, 7, device="cuda"))
