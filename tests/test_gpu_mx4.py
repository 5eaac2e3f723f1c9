"""MX4 quantisation, its reverse and the MX4 product against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import mx4_reference as R
import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _strided(x, pad, offset=0):
    """The same values as a view into a wider buffer whose other elements are NaN."""
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=x.dtype, device=x.device)
    v = wide[:, offset:offset + x.shape[1]]
    v.copy_(x)
    return v


def _check_quantized(x):
    codes, scales = P.mx4_quantize(x)
    want_c, want_s = R.quantize(x.double().cpu().numpy())
    got_c, got_s = codes.cpu().numpy(), scales.cpu().numpy()
    assert (got_s == want_s).all()
    fine = np.repeat(want_s != 255, 16, 1)                     # codes of a NaN block mean nothing
    assert (got_c[fine] == want_c[fine]).all()
    return codes, scales, want_c, want_s


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (3, 31, 0, 0), (2, 32, 0, 0), (5, 33, 3, 1), (7, 1024, 8, 8), (1, 4096, 0, 0),
                                                  (4, 1413, 11, 0), (130, 96, 0, 0), (3, 2049, 0, 0), (600, 64, 64, 0),
                                                  (700, 33, 7, 0), (41, 7, 1, 1), (333, 200, 8, 0), (35, 992, 0, 0), (34, 993, 31, 0), (65, 500, 4, 0), (1025, 1, 0, 0)])
def test_quantize_and_back(dt, rows, cols, pad, offset):
    g = _gen(rows * 7 + cols)
    x = torch.randn(rows, cols, generator=g) * torch.exp(2 * torch.randn(rows, 1, generator=g))
    x = x.to(DT[dt]).to(DEV)
    x = _strided(x, pad, offset) if pad else x
    codes, scales, want_c, want_s = _check_quantized(x)
    for out in ("f32", "bf16", "f16"):
        y = P.mx4_dequantize(codes, scales, cols, dtype=DT[out])
        want = torch.from_numpy(R.values(want_c, want_s)[:, :cols]).to(DT[out])   # exact, or one rounding
        assert torch.equal(y.cpu(), want)


def test_every_code_under_every_scale():
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1)            # 512 values = 16 blocks a row
    scales = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 16)
    for name, dt in DT.items():
        y = P.mx4_dequantize(codes.to(DEV), scales.to(DEV), 512, dtype=dt).cpu()
        with np.errstate(over="ignore"):
            want = torch.from_numpy(R.values(codes.numpy(), scales.numpy())).to(dt)
        assert torch.equal(y.isnan(), want.isnan()), name
        assert torch.equal(torch.nan_to_num(y, nan=7.0), torch.nan_to_num(want, nan=7.0)), name


def test_ties_saturation_signs_and_extremes():
    row = [0.25, -0.25, 0.75, -0.75, 1.25, 1.75, 2.5, -2.5, 3.5, -3.5, 5.0, -5.0, 7.99, -7.99, 6.0, 4.0]
    x = torch.zeros(8, 64)
    x[0, :16] = torch.tensor(row)
    x[1, :16] = torch.tensor(row) * 2.0 ** 100
    x[2, :16] = torch.tensor(row) * 2.0 ** -120
    x[3, :4] = torch.tensor([2.0 ** -149, -2.0 ** -149, 2.0 ** -130, 2.0 ** -127])   # below the smallest scale
    x[4, :3] = torch.tensor([torch.finfo(torch.float32).max, torch.finfo(torch.float32).min, 1.0])
    x[5] = -0.0
    x[6, 40] = 1.0                                                          # a block of zeros beside one that is not
    _check_quantized(x.to(DEV))


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_nan_and_infinity_poison_their_block_alone(dt):
    x = torch.randn(4, 160, generator=_gen(3)).to(DT[dt])
    x[0, 5], x[1, 64], x[2, 159], x[3, 32] = float("nan"), float("inf"), float("-inf"), float("nan")
    x[3, 33] = float("inf")
    codes, scales, _, want_s = _check_quantized(x.to(DEV))
    assert (want_s == 255).sum() == 4
    y = P.mx4_dequantize(codes, scales, 160)
    bad = torch.from_numpy(np.repeat(want_s == 255, 32, 1))
    assert torch.equal(y.isnan().cpu(), bad)


def test_given_outputs_with_strides_leave_their_neighbours():
    x = torch.randn(9, 80, generator=_gen(4), dtype=torch.float32).to(DEV)
    codes = torch.full((9, 64), 0xAA, dtype=torch.uint8, device=DEV)
    scales = torch.full((9, 7), 0xBB, dtype=torch.uint8, device=DEV)
    P.mx4_quantize(x, codes[:, 4:52], scales[:, 2:5])
    want_c, want_s = R.quantize(x.double().cpu().numpy())
    assert (codes[:, 4:52].cpu().numpy() == want_c).all() and (scales[:, 2:5].cpu().numpy() == want_s).all()
    assert (codes[:, :4] == 0xAA).all() and (codes[:, 52:] == 0xAA).all()
    assert (scales[:, :2] == 0xBB).all() and (scales[:, 5:] == 0xBB).all()
    out = torch.full((9, 90), 7.0, device=DEV)
    P.mx4_dequantize(codes[:, 4:52], scales[:, 2:5], 80, out=out[:, 3:83])
    assert (out[:, :3] == 7).all() and (out[:, 83:] == 7).all()
    assert (out[:, 3:83].double().cpu().numpy() == R.values(want_c, want_s)[:, :80]).all()


def test_no_rows():
    x = torch.empty(0, 64, device=DEV)
    codes, scales = P.mx4_quantize(x)
    assert codes.shape == (0, 32) and scales.shape == (0, 2)
    assert P.mx4_dequantize(codes, scales, 64).shape == (0, 64)
    w = P.mx4_quantize(torch.randn(16, 64, device=DEV))
    assert P.mx4_matmul((codes, scales), w).shape == (0, 16)


# ---- product -----------------------------------------------------------------------------------

def _operand(g, rows, nb, lo=126, hi=128):
    """Random codes under scales 2^-1 .. 2: every product is a multiple of 2^-4 below 144, so sums of
    up to 2^15 of them are exact in fp32 whatever the order."""
    codes = torch.randint(0, 256, (rows, nb * 16), generator=g, dtype=torch.uint8)
    scales = torch.randint(lo, hi + 1, (rows, nb), generator=g, dtype=torch.uint8)
    return codes, scales


def _product(a, b, counts=None):
    """fp64 [m][n]; rows that belong to no group are NaN."""
    va, vb = R.values(*[t.numpy() for t in a]), R.values(*[t.numpy() for t in b])
    if counts is None:
        return va @ vb.T
    out, at = np.full((va.shape[0], vb.shape[1]), np.nan), 0
    for g, c in enumerate(counts):
        out[at:at + c] = va[at:at + c] @ vb[g].T
        at += c
    return out


def _dev(pair):
    return tuple(t.to(DEV) for t in pair)


@pytest.mark.parametrize("m,n,nb", [(1, 16, 1), (1, 1, 1), (2, 129, 3), (16, 128, 8), (17, 128, 9), (5, 300, 64), (33, 64, 17), (64, 1000, 5),
                                    (65, 257, 8), (130, 128, 24), (128, 128, 16), (193, 130, 40), (500, 384, 12), (1, 19000, 8), (400, 2000, 33)])
def test_product_exact_sums(m, n, nb):
    g = _gen(m * 31 + n + nb)
    a, b = _operand(g, m, nb), _operand(g, n, nb)
    want = torch.from_numpy(_product(a, b))
    flags = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = P.mx4_matmul(_dev(a), _dev(b), dtype=torch.float32, flags=flags)
    assert flags.item() == 0
    assert torch.equal(got.double().cpu(), want)              # every sum is exact in fp32
    for dt in (torch.bfloat16, torch.float16):
        got = P.mx4_matmul(_dev(a), _dev(b), dtype=dt).cpu()
        assert torch.equal(got, want.float().to(dt))          # one rounding


@pytest.mark.parametrize("counts,n,nb", [([3, 0, 5, 1], 130, 4), ([0, 0, 0], 64, 2), ([70, 1, 0, 200, 33], 256, 9), ([0, 17], 100, 8),
                                         ([1] * 40, 140, 3), ([300, 300], 257, 5), ([2, 2], 2048, 64)])
@pytest.mark.parametrize("behind", [0, 7])
def test_product_by_group(counts, n, nb, behind):
    g = _gen(sum(counts) + n)
    m, E = sum(counts) + behind, len(counts)
    if m == 0:
        m = 1
    a = _operand(g, m, nb)
    bc, bs = _operand(g, E * n, nb)
    b = (bc.view(E, n, -1), bs.view(E, n, -1))
    want = torch.from_numpy(_product(a, b, counts))
    out = torch.full((m, n), 12345.0, device=DEV)
    P.mx4_matmul(_dev(a), _dev(b), counts=torch.tensor(counts, dtype=torch.int32, device=DEV), out=out)
    used = sum(counts)
    assert torch.equal(out[:used].double().cpu(), want[:used])
    assert (out[used:] == 12345.0).all()                      # rows without a group stay as they were


def test_product_with_counts_that_lead_past_the_rows():
    g = _gen(11)
    a = _operand(g, 20, 3)
    bc, bs = _operand(g, 4 * 50, 3)
    b = (bc.view(4, 50, -1), bs.view(4, 50, -1))
    out = P.mx4_matmul(_dev(a), _dev(b), counts=torch.tensor([5, -3, 40, 2 ** 31 - 1], dtype=torch.int32, device=DEV), dtype=torch.float32)
    assert torch.equal(out.double().cpu(), torch.from_numpy(_product(a, b, [5, 0, 15, 0])))


@pytest.mark.parametrize("m,n,k", [(3, 200, 100), (150, 130, 1000), (40, 64, 4096)])
def test_product_of_quantized_values(m, n, k):
    g = _gen(m + n + k)
    x = torch.randn(m, k, generator=g)
    w = 0.02 * torch.randn(n, k, generator=g)
    a, b = P.mx4_quantize(x.bfloat16().to(DEV)), P.mx4_quantize(w.to(DEV))
    got = P.mx4_matmul(a, b, dtype=torch.float32).double().cpu()
    va, vb = (R.values(c.cpu().numpy(), s.cpu().numpy()) for c, s in (a, b))
    # exact products; k - 1 fp32 additions in any order, each off by at most 2^-23 of the sum of magnitudes
    # (a truncating adder; a rounding one is off by half of that)
    bound = torch.from_numpy(k * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T))
    assert ((got - torch.from_numpy(va @ vb.T)).abs() <= bound).all()


def test_product_strides_and_wide_scale_range():
    g = _gen(21)
    m, n, nb = 37, 150, 11
    a, b = _operand(g, m, nb, 60, 61), _operand(g, n, nb, 190, 191)   # 2^-67.. times 2^63..: sums still exact
    ac = torch.zeros(m, nb * 16 + 48, dtype=torch.uint8, device=DEV)
    as_ = torch.full((m, nb + 5), 255, dtype=torch.uint8, device=DEV)
    bc = torch.full((n, nb * 16 + 16), 0x77, dtype=torch.uint8, device=DEV)
    bs = torch.full((n, nb + 3), 255, dtype=torch.uint8, device=DEV)
    av, asv, bv, bsv = ac[:, 16:16 + nb * 16], as_[:, 3:3 + nb], bc[:, :nb * 16], bs[:, 1:1 + nb]
    av.copy_(a[0]), asv.copy_(a[1]), bv.copy_(b[0]), bsv.copy_(b[1])
    out = torch.full((m, n + 9), 5.0, device=DEV)
    P.mx4_matmul((av, asv), (bv, bsv), out=out[:, 4:4 + n])
    assert torch.equal(out[:, 4:4 + n].double().cpu(), torch.from_numpy(_product(a, b)))
    assert (out[:, :4] == 5).all() and (out[:, 4 + n:] == 5).all()


def test_product_nan_blocks_reach_their_rows_alone():
    g = _gen(22)
    a, b = _operand(g, 20, 9), _operand(g, 140, 9)
    a[1][7, 8], b[1][130, 0] = 255, 255
    got = P.mx4_matmul(_dev(a), _dev(b), dtype=torch.float32).cpu()
    bad = torch.zeros(20, 140, dtype=torch.bool)
    bad[7], bad[:, 130] = True, True
    assert torch.equal(got.isnan(), bad)
    a[1][7, 8], b[1][130, 0] = 127, 127
    want = torch.from_numpy(_product(a, b))
    assert torch.equal(got[~bad].double(), want[~bad])


def test_product_on_another_stream_and_replayed():
    g = _gen(23)
    a, b = _dev(_operand(g, 24, 40)), _dev(_operand(g, 512, 40))
    want = P.mx4_matmul(a, b)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = P.mx4_matmul(a, b, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    x = torch.randn(24, 1280, generator=_gen(1)).to(DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = P.mx4_matmul(P.mx4_quantize(x), b)
    for seed in (2, 3):
        x.copy_(torch.randn(24, 1280, generator=_gen(seed)))
        graph.replay()
        assert torch.equal(y, P.mx4_matmul(P.mx4_quantize(x), b))


# ---- sizes whose offsets pass 32 bits ------------------------------------------------------------

def test_quantize_and_back_behind_four_billion_elements():
    """70000 x 65536 bf16 (9 GB): elements, and with a row of padding bytes too, beyond 2^32."""
    rows, cols = 70000, 65536
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    x[:8].normal_()
    x[8:] = 1.0
    x[-4:] = x[:4]
    x[rows // 2] = x[5]
    codes, scales = P.mx4_quantize(x)
    few_c, few_s = P.mx4_quantize(x[:8].clone())
    for big, few in ((slice(0, 8), slice(0, 8)), (slice(rows - 4, rows), slice(0, 4)), (slice(rows // 2, rows // 2 + 1), slice(5, 6))):
        assert torch.equal(codes[big], few_c[few]) and torch.equal(scales[big], few_s[few])
    del x
    y = P.mx4_dequantize(codes, scales, cols, dtype=torch.bfloat16)
    z = P.mx4_dequantize(few_c, few_s, cols, dtype=torch.bfloat16)
    assert torch.equal(y[-4:], z[:4]) and torch.equal(y[rows // 2], z[5])
    del y
    wide = torch.empty(rows, 65540, dtype=torch.bfloat16, device=DEV)[:, :cols]   # rows off the 16-byte grid
    P.mx4_dequantize(codes, scales, cols, out=wide)
    assert torch.equal(wide[-4:], z[:4]) and torch.equal(wide[:8], z)


def test_product_with_more_than_two_billion_outputs():
    m, n, nb = 40003, 60001, 1
    g = _gen(41)
    a, b = _operand(g, m, nb), _operand(g, n, nb)
    out = P.mx4_matmul(_dev(a), _dev(b), dtype=torch.bfloat16)
    rows = [0, 1, 17777, 35791, 35792, m - 2, m - 1]          # 35792 * 60001 passes 2^31
    want = _product([t[rows] for t in a], b)
    assert torch.equal(out[rows].cpu(), torch.from_numpy(want).float().bfloat16())


@pytest.mark.parametrize("blocks", [16, 12, 35])   # scale rows on 8, 4 and 1 bytes: a read path each
def test_chain_through_the_same_buffers_sees_each_step_s_values(blocks):
    """Each product reads what the quantisation just before it wrote over the last step's operand."""
    g = torch.Generator(device="cuda").manual_seed(blocks)
    rows, n, cols, steps = 700, 256, blocks * 32, 24
    xs = torch.randn(steps, rows, cols, device="cuda", generator=g, dtype=torch.bfloat16)
    b = P.mx4_quantize(torch.randn(n, cols, device="cuda", generator=g))
    want_x, want_y = [], []
    for x in xs:   # operands of their own, one step at a time
        q = P.mx4_quantize(x)
        torch.cuda.synchronize()
        want_x.append(P.mx4_dequantize(*q, cols))
        want_y.append(P.mx4_matmul(q, b))
        torch.cuda.synchronize()
    codes = torch.empty(rows, blocks * 16, dtype=torch.uint8, device="cuda")
    scales = torch.empty(rows, blocks, dtype=torch.uint8, device="cuda")
    back = torch.empty(steps, rows, cols, device="cuda")
    out = torch.empty(steps, rows, n, dtype=torch.bfloat16, device="cuda")
    for i, x in enumerate(xs):
        P.mx4_quantize(x, codes, scales)
        P.mx4_matmul((codes, scales), b, out=out[i])
        P.mx4_quantize(x.flip(0).contiguous(), codes, scales)
        P.mx4_dequantize(codes, scales, cols, out=back[i])
    assert all(torch.equal(out[i], want_y[i]) for i in range(steps))
    assert all(torch.equal(back[i], want_x[i].flip(0)) for i in range(steps))
