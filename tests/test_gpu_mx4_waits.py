"""Bounded waits of the MX4 kernels that run out, by a lowered poll limit (no barrier is broken: the limit
alone ends the waits): the kernels end, what depends on an expired wait is NaN, the rest is as it should be, and the
next call with the default limit is whole."""
import pytest
import torch

import paper_2606_15453_b200 as P
from paper_2606_15453_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DEFAULT = 1 << 22


@pytest.fixture
def polls():
    yield binding.mx4_poll_limit
    torch.cuda.synchronize()
    binding.mx4_poll_limit(DEFAULT)


def _rows(g, rows, nb):
    return (torch.randint(0, 256, (rows, nb * 16), generator=g, device=DEV, dtype=torch.uint8),
            torch.randint(126, 129, (rows, nb), generator=g, device=DEV, dtype=torch.uint8))


def _product(seed, counts, behind, n, nb, dt, pad):
    g = torch.Generator(device=DEV).manual_seed(seed)
    E, m = len(counts), sum(counts) + behind
    bc, bs = _rows(g, E * n, nb)
    a, b = _rows(g, m, nb), (bc.view(E, n, -1), bs.view(E, n, -1))
    cd = torch.tensor(counts, dtype=torch.int32, device=DEV)
    out = torch.full((m, n + pad), 7.0, dtype=dt, device=DEV)[:, :n]

    def call():
        out.fill_(7.0)
        flags = torch.zeros(1, dtype=torch.int32, device=DEV)
        P.mx4_matmul(a, b, counts=cd, out=out, flags=flags)
        torch.cuda.synchronize()
        return out.clone(), flags.item()
    return call, sum(counts)


# a tile or more for every CTA, whole lines of the output and not; a reduction split over clusters; groups
PRODUCTS = [([700], 0, 40000, 9, torch.bfloat16, 0), ([700], 3, 40001, 9, torch.float32, 0), ([300, 0, 41], 5, 20000, 12, torch.float16, 8),
            ([5], 2, 512, 64, torch.bfloat16, 0), ([3, 4], 0, 200, 24, torch.float32, 1)]


@pytest.mark.parametrize("case", range(len(PRODUCTS)))
def test_product_whose_waits_give_up_at_once_is_nan_throughout(polls, case):
    call, used = _product(case, *PRODUCTS[case])
    want, flag = call()
    assert flag == 0 and want[:used].isfinite().all()
    polls(0)
    got, flag = call()
    assert flag == 1 and got[:used].isnan().all() and (got[used:] == 7).all()
    polls(DEFAULT)
    again, flag = call()
    assert flag == 0 and torch.equal(again, want)


@pytest.mark.parametrize("limit", [1, 2, 4, 8])
@pytest.mark.parametrize("case", range(len(PRODUCTS)))
def test_product_whose_waits_give_up_on_the_way_is_whole_or_nan(polls, case, limit):
    """A few polls, some microseconds each: some waits hold and some run out, with loads and MMAs under way."""
    call, used = _product(case, *PRODUCTS[case])
    want, _ = call()
    polls(limit)
    for _ in range(3):
        got, flag = call()
        bad = got[:used].isnan()
        assert torch.equal(got[:used][~bad], want[:used][~bad]) and (got[used:] == 7).all()
        assert flag == 1 or not bad.any()
    polls(DEFAULT)
    again, flag = call()
    assert flag == 0 and torch.equal(again, want)
