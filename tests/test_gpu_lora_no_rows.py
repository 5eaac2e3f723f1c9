"""The gradients of adapters that nobody used, through the C entry: a step without rows clears them, right behind a grouping that
still writes its counts over those of the step before."""
import pytest
import torch

import paper_2606_15453_b200 as P
from paper_2606_15453_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("which", ["both", "a", "b", "none"])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,r,I,O", [(1, 1, 1, 1), (5, 16, 520, 264), (300, 3, 33, 17)])
def test_gradients_of_a_step_without_rows(n, r, I, O, dt, which):
    L, i32 = P.lib(), torch.int32
    x, g, dx = (torch.zeros(1, c, dtype=dt, device=DEV) for c in (I, O, I))     # not read, but an address
    a, b = torch.ones(n, r, I, dtype=dt, device=DEV), torch.ones(n, O, r, dtype=dt, device=DEV)
    hidden = torch.zeros(1, device=DEV)
    some = torch.zeros(1, dtype=i32, device=DEV)
    size = L.stmoe_lora_backward_scratch_bytes(0, n, r, I, O)
    scratch = torch.empty(size + 256, dtype=torch.uint8, device=DEV)
    elem, st = binding._ELEM[dt], torch.cuda.current_stream().cuda_stream
    at = (scratch.data_ptr() + 255) // 256 * 256
    for _ in range(20):
        counts, starts = torch.full((n,), 100000, dtype=i32, device=DEV), torch.full((n + 1,), 100000, dtype=i32, device=DEV)
        da, db = torch.full((n, r, I), 7., dtype=dt, device=DEV), torch.full((n, O, r), 7., dtype=dt, device=DEV)
        assert L.stmoe_group_rows(some.data_ptr(), 0, 1, n, counts.data_ptr(), starts.data_ptr(), some.data_ptr(), some.data_ptr(), None, 0, st) == 0
        assert L.stmoe_lora_backward(g.data_ptr(), elem, O, x.data_ptr(), I, 0, a.data_ptr(), r * I, I, b.data_ptr(), O * r, r, n, r, I, O,
                                     some.data_ptr(), some.data_ptr(), counts.data_ptr(), starts.data_ptr(), None, 1.0, hidden.data_ptr(), dx.data_ptr(), I,
                                     da.data_ptr() if which in ("both", "a") else None, db.data_ptr() if which in ("both", "b") else None, at, size, st) == 0
        torch.cuda.synchronize()
        assert not counts.any() and not starts.any()
        assert (da == (0 if which in ("both", "a") else 7)).all() and (db == (0 if which in ("both", "b") else 7)).all()
