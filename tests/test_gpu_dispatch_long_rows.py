"""Dispatch of rows as long as the call takes: 2^31 - 1 bytes, in units of one byte and of wider ones."""
import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype,cols", [(torch.uint8, 2 ** 31 - 1), (torch.uint8, 2 ** 31 - 128), (torch.uint8, 2 ** 30 + 1), (torch.float16, 2 ** 30 - 1), (torch.float32, 2 ** 29 - 4)])
def test_rows_of_two_gigabytes(dtype, cols):
    g = torch.Generator(device=DEV).manual_seed(1)
    noise = torch.randint(0, 256, (2 ** 20 + 77,), dtype=torch.uint8, generator=g, device=DEV)
    size = torch.empty(0, dtype=dtype).element_size()
    x = noise.repeat(-(-2 * cols * size // noise.numel()))[:2 * cols * size].view(dtype).view(2, cols)
    ids = torch.tensor([[1, 0], [-1, 0]], dtype=torch.int32, device=DEV)      # three rows in groups, and one behind them
    out = P.dispatch_rows(x, P.group_rows(ids, 2))
    want = [x[0], x[1], x[0]]
    for got, w in zip(out, want):
        assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))
    assert not out[3].view(torch.uint8).any()
