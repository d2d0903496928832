"""4-bit microscaled rows and their product on the GPU against the definitions in 64 bits.

Quantizing and reading back have one right answer.  A product's bound: the bf16 output is at most half a unit off, 2^-8 of
its magnitude, and K fp32 additions, each taken as truncating (2^-23), are off by at most K * 2^-23 of the sum of magnitudes."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu


def _rows(seed, rows, cols, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g)
    if kind == "wide":                      # every exponent a bf16 number has, zeros and subnormals among them
        x = torch.randint(0, 0x7f80, (rows, cols), generator=g).to(torch.int16).view(torch.bfloat16).float()
        x *= torch.randint(0, 2, (rows, cols), generator=g) * 2 - 1
    elif kind == "ties":                    # multiples of a quarter of the scale: every tie there is
        x = torch.randint(-32, 33, (rows, cols), generator=g) / 4
        x[:, ::32] = 7.5
        x *= torch.exp2(torch.randint(-100, 100, (rows, 1), generator=g).float())
    return x.to(torch.bfloat16)


def _quantize(x):
    codes, scales = eq.alloc_mx4(*x.shape)
    codes.fill_(0xA5)
    scales.fill_(0x5A)
    eq.equarx_mx4_quantize(x, codes, scales)
    return codes, scales


@pytest.mark.parametrize("kind", ("normal", "wide", "ties"))
@pytest.mark.parametrize("rows,cols", ((1, 1), (1, 32), (3, 127), (5, 128), (2, 129), (7, 1511), (64, 5376), (1, 40001)))
def test_quantize_and_read_back(rows, cols, kind):
    x = _rows(rows + cols, rows, cols, kind)
    codes, scales = _quantize(x.cuda())
    want_codes, want_scales = ref.mx4_quantize(x)
    assert (scales.cpu().numpy() == want_scales).all()
    assert (codes.cpu().numpy() == want_codes).all()
    out = torch.full((rows, cols + 3), 9.0, dtype=torch.bfloat16, device="cuda")
    eq.equarx_mx4_dequantize(codes, scales, out[:, :cols])
    assert (out[:, :cols].double().cpu().numpy() == ref.mx4_values(want_codes, want_scales, cols)).all()
    assert (out[:, cols:] == 9.0).all()


@pytest.mark.parametrize("gap", (0, 1, 3, 8, 128))
def test_rows_of_any_stride_and_start(gap):
    wide = _rows(3, 37, 200 + gap).cuda()
    x = wide[:, gap // 8 * 8:gap // 8 * 8 + 200]
    codes, scales = _quantize(x)
    want_codes, want_scales = ref.mx4_quantize(x.cpu())
    assert (codes.cpu().numpy() == want_codes).all() and (scales.cpu().numpy() == want_scales).all()


def test_every_code_at_every_scale_reads_back():
    codes = torch.arange(16, dtype=torch.uint8).repeat(256, 4)
    codes = codes[:, 0::2] | codes[:, 1::2] << 4                    # 32 codes: each twice
    codes = codes.repeat(1, 2)                                      # two blocks, padded to a group below
    scales = torch.arange(256, dtype=torch.uint8).reshape(-1, 1).repeat(1, 4)
    codes = torch.cat((codes, torch.zeros(256, 64 - codes.shape[1], dtype=torch.uint8)), dim=1).contiguous()
    out = torch.empty(256, 128, dtype=torch.bfloat16, device="cuda")
    eq.equarx_mx4_dequantize(codes.cuda(), scales.cuda(), out)
    got, want = out.double().cpu().numpy(), ref.mx4_values(codes.numpy(), scales.numpy(), 128)
    biggest = float(torch.finfo(torch.bfloat16).max)
    want = np.where(np.abs(want) > biggest, np.sign(want) * np.inf, want)       # 2^127 * 2 and more: beyond bf16
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("bad", (float("nan"), float("inf"), -float("inf")))
def test_a_block_that_is_not_finite_reads_back_as_nan(bad):
    x = _rows(5, 3, 300)
    x[1, 70] = bad
    codes, scales = _quantize(x.cuda())
    out = torch.empty(3, 300, dtype=torch.bfloat16, device="cuda")
    eq.equarx_mx4_dequantize(codes, scales, out)
    hit = torch.zeros(3, 300, dtype=torch.bool)
    hit[1, 64:96] = True
    assert torch.equal(torch.isnan(out).cpu(), hit)
    w = _quantize(_rows(6, 17, 300).cuda())
    for xs, ws, where in (((codes, scales), w, (1, slice(None))), (w, (codes, scales), (slice(None), 1))):
        got = torch.empty(xs[0].shape[0], ws[0].shape[0], dtype=torch.bfloat16, device="cuda")
        eq.equarx_mx4_product(*xs, *ws, 300, got, eq.alloc_mx4_workspace(*got.shape, 300))
        want = torch.zeros(got.shape, dtype=torch.bool)
        want[where] = True
        assert torch.equal(torch.isnan(got).cpu(), want)


def _bound(x, w, want):
    return 2.0 ** -8 * want.abs() * (1 + 2.0 ** -8) + (x.shape[1] + 8) * 2.0 ** -23 * (x.abs() @ w.abs().T) + 2.0 ** -133


SHAPES = [(1, 1, 1), (1, 16, 128), (1, 5376, 257), (2, 33, 4096), (15, 100, 640), (16, 17, 129), (17, 250, 1511), (48, 64, 384),
          (63, 129, 512), (64, 320, 1024), (65, 1000, 130), (100, 31, 2048), (127, 255, 767), (128, 128, 256), (129, 257, 1025),
          (200, 515, 640), (256, 256, 1024), (257, 129, 2000), (300, 1030, 300), (512, 512, 128), (640, 384, 4096)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product_and_linear(M, N, K):
    x, w = _rows(M, M, K).cuda(), (_rows(N + 1, N, K) * K ** -0.5).cuda()
    xq, wq = _quantize(x), _quantize(w)
    xv, wv = (torch.from_numpy(ref.mx4_values(c.cpu().numpy(), s.cpu().numpy(), K)) for c, s in (xq, wq))
    want = xv @ wv.T
    gap = 5
    out = torch.full((M, N + gap), 9.0, dtype=torch.bfloat16, device="cuda")
    work = eq.alloc_mx4_workspace(M, N, K)
    work.fill_(0xFF)                        # nothing in it needs clearing
    eq.equarx_mx4_product(*xq, *wq, K, out[:, :N], work)
    assert ((out[:, :N].double().cpu() - want).abs() <= _bound(xv, wv, want)).all()
    assert (out[:, N:] == 9.0).all()
    again = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda")
    work.fill_(0xFF)
    eq.equarx_mx4_linear(x, *wq, again, work)
    assert torch.equal(again, out[:, :N])


# One shape for each kernel and tile there is (32 x 32, 64 and 128 rows; 128 x 64; 128 x 128 alone on a CU and in pairs; 256 x 256), none
# a whole number of tiles, with every remainder that k's groups can leave.
TILES = [(9, 77), (50, 77), (100, 1000), (300, 1100), (600, 4100), (1100, 4130), (2111, 4101)]


@pytest.mark.parametrize("M,N", TILES)
@pytest.mark.parametrize("groups", (1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 15, 21))
def test_every_tile_with_every_remainder_of_k(M, N, groups):
    K = groups * 128 - 37
    g = torch.Generator(device="cuda").manual_seed(groups)
    x, w = (torch.randn(n, K, generator=g, device="cuda").to(torch.bfloat16) for n in (M, N))
    xq, wq = _quantize(x), _quantize(w)
    values = []
    for codes, scales in (xq, wq):
        v = torch.empty(codes.shape[0], K, dtype=torch.bfloat16, device="cuda")
        eq.equarx_mx4_dequantize(codes, scales, v)
        values.append(v.double())
    want = values[0] @ values[1].T.contiguous()
    out = torch.full((M, N), 9.0, dtype=torch.bfloat16, device="cuda")
    eq.equarx_mx4_product(*xq, *wq, K, out, eq.alloc_mx4_workspace(M, N, K))
    assert ((out.double() - want).abs() <= _bound(*values, want)).all()


def test_linear_takes_rows_of_any_stride():
    for gap in (1, 8):
        wide = _rows(9, 21, 700 + gap).cuda()
        x, w = wide[:, :700], _quantize(_rows(10, 90, 700).cuda())
        outs = [torch.empty(21, 90, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        work = eq.alloc_mx4_workspace(21, 90, 700)
        eq.equarx_mx4_linear(x, *w, outs[0], work)
        eq.equarx_mx4_linear(x.contiguous(), *w, outs[1], work)
        assert torch.equal(*outs)


def test_a_product_over_nothing_is_zero():
    lib = eq.load()
    out = torch.full((5, 40), 9.0, dtype=torch.bfloat16, device="cuda")
    assert lib.equarx_mx4_product(None, None, None, None, 5, 40, 0, out.data_ptr(), 40, None, 0, eq._stream()) == 0
    assert (out == 0).all()


def test_scales_at_the_ends_of_their_range():
    """Products of a small and a large scale are as exact as any."""
    for up, down in ((120, -120), (-126, 126), (60, -126)):
        x, w = _rows(11, 20, 256).float() * 2.0 ** up, _rows(12, 50, 256).float() * 2.0 ** down
        xq, wq = _quantize(x.to(torch.bfloat16).cuda()), _quantize(w.to(torch.bfloat16).cuda())
        xv, wv = (torch.from_numpy(ref.mx4_values(c.cpu().numpy(), s.cpu().numpy(), 256)) for c, s in (xq, wq))
        out = torch.empty(20, 50, dtype=torch.bfloat16, device="cuda")
        eq.equarx_mx4_product(*xq, *wq, 256, out, eq.alloc_mx4_workspace(20, 50, 256))
        want = xv @ wv.T
        assert ((out.double().cpu() - want).abs() <= _bound(xv, wv, want)).all(), (up, down)


def test_on_another_stream_and_in_a_graph():
    x, w = _rows(13, 40, 900).cuda(), _quantize(_rows(14, 300, 900).cuda())
    work = eq.alloc_mx4_workspace(40, 300, 900)
    want, out = (torch.zeros(40, 300, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    eq.equarx_mx4_linear(x, *w, want, work)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        eq.equarx_mx4_linear(x, *w, out, work)
    stream.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eq.equarx_mx4_linear(x, *w, out, work)
    for seed in (15, 16, 17):
        x.copy_(_rows(seed, 40, 900))
        eq.equarx_mx4_linear(x, *w, want, work)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
