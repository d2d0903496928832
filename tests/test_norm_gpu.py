"""Root-mean-square norms on the GPU against the definition.

The row's mean is a sum of at most 2^15 exact squares in 64 bits, off by at most 2^15 * 2^-53 of itself, and its inverse root by half of
that and a few 2^-53: less than 2^-37.  So the factor is the fp32 number that the exact one rounds to, or, where that is nearer than
2^-36 to a border, the one on its other side; every product after it is rounded where the definition says so.  A row's outputs are those
of one of the two, bit for bit; for all rows but a few in 2^12 they are the same."""
import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu


def _rows(seed, rows, cols, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g)
    if kind == "spread":
        x *= torch.exp2(torch.randint(-60, 60, (rows, 1), generator=g).float())
    return x.to(torch.bfloat16)


def _two(x, weight, eps, residual=None, one_plus=False):
    """h (bf16) and y (fp32) with either factor."""
    h = x if residual is None else (x.float() + residual.float()).to(torch.bfloat16)
    exact = 1.0 / np.sqrt(np.square(h.double().numpy()).sum(axis=1) / h.shape[1] + eps)
    g = None if weight is None else (weight.float() + 1.0 if one_plus else weight.float())
    ys = []
    for side in (1 - 2.0 ** -36, 1 + 2.0 ** -36):
        y = h.float() * torch.from_numpy((exact * side).astype(np.float32))[:, None]
        ys.append(y if g is None else y * g)
    return h, ys


def _int8(y, block):
    w = y.reshape(-1, block)
    finite = torch.isfinite(w).all(dim=1, keepdim=True)
    w = torch.where(finite, w, 0.0)
    top = w.abs().amax(dim=1, keepdim=True)
    alive = top >= 127 * 2.0 ** -126
    most = torch.full_like(top, 127.0)                              # quotients of tensors: torch takes a number's by a reciprocal
    scale = torch.where(alive, top / most, 0.0)
    codes = torch.round(w * torch.where(alive, most / torch.where(alive, top, 1.0), 0.0))
    return codes.to(torch.int8).reshape(y.shape), torch.where(finite, scale, float("nan")).reshape(y.shape[0], -1)


def _rows_match(got, wants):
    """Every row of `got` has the bits of that row of one of `wants`; NaN is NaN."""
    def same(want):
        eq_ = got == want
        if got.is_floating_point():
            eq_ |= got.isnan() & want.isnan()
            if got.dtype != torch.float64:
                eq_ &= (got.signbit() == want.signbit()) | got.isnan()
        return eq_.reshape(got.shape[0], -1).all(dim=1)
    ok = same(wants[0]) | same(wants[1])
    assert ok.all(), (~ok).nonzero().flatten()[:8].tolist()


def _run(x, weight, eps=1e-6, residual=None, one_plus=False, block=0, mx4=False, out=True, stream_shape=None):
    rows, cols = x.shape
    pad = lambda t: torch.full((rows, t.shape[1] + 5), 9.0, dtype=torch.bfloat16, device="cuda")
    results = {}
    kw = {}
    if out:
        results["wide"] = torch.full((rows, cols + 3), 9.0, dtype=torch.bfloat16, device="cuda")
        kw["out"] = results["wide"][:, :cols]
    if block:
        kw.update(codes=torch.full((rows, cols), 77, dtype=torch.int8, device="cuda"),
                  scales=torch.full((rows, cols // block), 7.0, device="cuda"), codes_block=block)
    if mx4:
        codes, scales = eq.alloc_mx4(rows, cols)
        codes.fill_(0xA5), scales.fill_(0x5A)
        kw.update(mx4_codes=codes, mx4_scales=scales)
    if residual is not None:
        results["stream"] = pad(residual)
        results["stream"][:, :cols] = residual.cuda()
        kw["residual"] = results["stream"][:, :cols]
    eq.equarx_norm(x if x.is_cuda else x.cuda(), None if weight is None else weight.cuda(), eps, one_plus=one_plus, **kw)
    return results, kw


def _check(x, weight, eps=1e-6, residual=None, one_plus=False, block=0, mx4=False, out=True):
    results, kw = _run(x, weight, eps, residual, one_plus, block, mx4, out)
    rows, cols = x.shape
    h, ys = _two(x.cpu(), weight, eps, residual, one_plus)
    if residual is not None:
        stream = results["stream"].cpu()
        _rows_match(stream[:, :cols], (h, h))
        assert (stream[:, cols:] == 9.0).all()
    if out:
        wide = results["wide"].cpu()
        _rows_match(wide[:, :cols], [y.to(torch.bfloat16) for y in ys])
        assert (wide[:, cols:] == 9.0).all()
    if block:
        wants = [_int8(y, block) for y in ys]
        _rows_match(torch.cat((kw["codes"].cpu().double(), kw["scales"].cpu().double()), dim=1),
                    [torch.cat((c.double(), s.double()), dim=1) for c, s in wants])
    if mx4:
        wants = [tuple(torch.from_numpy(t) for t in ref.mx4_quantize(y)) for y in ys]
        _rows_match(torch.cat((kw["mx4_codes"].cpu(), kw["mx4_scales"].cpu()), dim=1), [torch.cat(w, dim=1) for w in wants])


SIZES = ((1, 1), (1, 7), (3, 8), (5, 33), (130, 127), (70, 128), (33, 129), (9, 511), (4, 512), (6, 513), (3, 1024), (2, 1031), (7, 2048),
         (3, 2049), (2, 4096), (1, 4097), (5, 5376), (64, 5376), (2, 6145), (3, 8192), (2, 8193), (3, 16384), (2, 16391), (2, 32768), (1, 32765))


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("residual", (False, True))
def test_bf16_and_packed_rows(rows, cols, residual):
    w = (1 + 0.2 * torch.randn(cols, generator=torch.Generator().manual_seed(1))).to(torch.bfloat16)
    _check(_rows(rows * 7 + cols, rows, cols, "spread"), w, residual=_rows(cols, rows, cols, "spread") if residual else None, mx4=True)


@pytest.mark.parametrize("block", (32, 64, 128, 256, 512))
@pytest.mark.parametrize("rows,blocks", ((1, 1), (67, 1), (5, 3), (3, 8), (2, 10), (2, 16), (65, 21), (1, 64)))
def test_int8_rows(block, rows, blocks):
    cols = min(block * blocks, 32768 // block * block)
    w = (1 + 0.2 * torch.randn(cols, generator=torch.Generator().manual_seed(2))).to(torch.bfloat16)
    _check(_rows(rows + cols, rows, cols), w, residual=_rows(cols, rows, cols), block=block, mx4=rows % 2 == 1)


@pytest.mark.parametrize("cols", (96, 1500, 5376))
@pytest.mark.parametrize("weight,one_plus", ((None, False), (0.1, True), (1.0, False)))
def test_weights(cols, weight, one_plus):
    w = None if weight is None else (weight * torch.randn(cols, generator=torch.Generator().manual_seed(3))).to(torch.bfloat16)
    _check(_rows(5, 9, cols), w, eps=0.3, one_plus=one_plus, mx4=True, block=0)


@pytest.mark.parametrize("cols", (64, 300, 2048))
def test_weights_of_every_size(cols):
    """Products down to subnormal numbers and zero, and up to infinity."""
    g = torch.Generator().manual_seed(4)
    w = torch.randint(0, 0x7f80, (cols,), generator=g).to(torch.int16).view(torch.bfloat16)
    w[::3] = -w[::3]
    _check(_rows(6, 11, cols), w, mx4=True, block=64 if cols % 64 == 0 else 0)


@pytest.mark.parametrize("eps", (0.0, 1e-6, 3.0))
def test_rows_of_zeros_and_of_the_smallest_and_largest(eps):
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    x[1] = torch.tensor([1], dtype=torch.int16).view(torch.bfloat16)             # 2^-133
    x[2] = torch.finfo(torch.bfloat16).max
    x[3, 100] = -0.0
    x[3, 5] = 1.0
    results, kw = _run(x, None, eps)
    h, ys = _two(x, None, eps)
    _rows_match(results["wide"].cpu()[:, :256], [y.to(torch.bfloat16) for y in ys])
    assert (results["wide"][0, :256].isnan().all() if eps == 0 else (results["wide"][0, :256] == 0).all())


@pytest.mark.parametrize("bad", (float("nan"), float("inf"), -float("inf")))
@pytest.mark.parametrize("cols", (128, 640, 5376))
def test_a_row_that_is_not_finite_says_so_and_no_other_does(bad, cols):
    x = _rows(8, 21, cols)
    x[7, cols // 2] = bad
    _check(x, None, block=32, mx4=True)
    _check(x, None, residual=_rows(9, 21, cols), block=128, mx4=True)


@pytest.mark.parametrize("gap,cols", ((1, 200), (3, 2501), (8, 5376), (200, 200)))
def test_rows_of_any_stride(gap, cols):
    wide = _rows(3, 37, cols + gap).cuda()
    x = wide[:, gap // 8 * 8:gap // 8 * 8 + cols]
    w = _rows(4, 1, cols)[0]
    _check(x, w, residual=_rows(5, 37, cols), mx4=True)


@pytest.mark.parametrize("cols", (64, 999, 5376, 20000))
def test_in_place(cols):
    x, w = _rows(11, 50, cols), _rows(12, 1, cols)[0]
    at, separate = x.cuda(), torch.empty(50, cols, dtype=torch.bfloat16, device="cuda")
    eq.equarx_norm(at.clone(), w.cuda(), out=separate)
    eq.equarx_norm(at, w.cuda(), out=at)
    assert torch.equal(at, separate)


def test_more_rows_than_workgroups_of_one_launch():
    """2^20 workgroups of sixteen rows, and some: every input and output goes on where the first launch ends."""
    rows, cols = (16 << 20) + 37, 32
    g = torch.Generator("cuda").manual_seed(1)
    partials = [torch.randn(rows, cols, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)]
    x = torch.empty_like(partials[0])
    eq.equarx_reduce_fused([p.view(-1) for p in partials], 32, x.view(-1))

    def outputs(n):
        codes, scales = eq.alloc_mx4(n, cols)
        return dict(out=torch.full((n, cols), 9.0, dtype=torch.bfloat16, device="cuda"), codes=torch.full((n, cols), 99, dtype=torch.int8, device="cuda"),
                    scales=torch.full((n, 1), 9.0, device="cuda"), codes_block=32, mx4_codes=codes, mx4_scales=scales)

    for reduced in (False, True):
        stream = torch.ones_like(x)
        all_rows = outputs(rows)
        if reduced:
            eq.equarx_norm_reduced(partials, 32, None, residual=stream, **all_rows)
        else:
            eq.equarx_norm(x, None, residual=stream, **all_rows)
        for part in (slice(0, 64), slice((16 << 20) - 32, rows)):
            small, few = torch.ones_like(x[part]), outputs(x[part].shape[0])
            eq.equarx_norm(x[part], None, residual=small, **few)
            assert torch.equal(stream[part], small)
            for k, t in few.items():
                assert not torch.is_tensor(t) or torch.equal(all_rows[k][part], t), k
        assert not (all_rows["out"] == 9.0).all(dim=1).any() and not (all_rows["codes"] == 99).all(dim=1).any()
    _, ys = _two(x[-50:].cpu(), None, 1e-6, residual=torch.ones(50, cols, dtype=torch.bfloat16))
    _rows_match(all_rows["out"][-50:].cpu(), [y.to(torch.bfloat16) for y in ys])


def test_offsets_past_32_bits():
    cols, rows = 32768, 66000                                   # 2^31 elements are passed at row 65536
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[65500:] = torch.randn(500, cols, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).to(torch.bfloat16)
    stream = x.clone()
    packed = eq.alloc_mx4(rows, cols)
    codes, scales = torch.empty(rows, cols, dtype=torch.int8, device="cuda"), torch.empty(rows, cols // 256, device="cuda")
    eq.equarx_norm(x, None, residual=stream, out=x, codes=codes, scales=scales, codes_block=256, mx4_codes=packed[0], mx4_scales=packed[1])
    part = slice(65990, rows)
    small = stream[part].clone()
    alone = torch.empty_like(small)
    few = eq.alloc_mx4(10, cols)
    c, s = torch.empty(10, cols, dtype=torch.int8, device="cuda"), torch.empty(10, cols // 256, device="cuda")
    eq.equarx_norm(small, None, out=alone, codes=c, scales=s, codes_block=256, mx4_codes=few[0], mx4_scales=few[1])
    assert alone.abs().max() > 1 and torch.equal(x[part], alone)
    assert torch.equal(codes[part], c) and torch.equal(scales[part], s)
    assert torch.equal(packed[0][part], few[0]) and torch.equal(packed[1][part], few[1])


# ---------------------------------------------------------------- norms of a reduction

@pytest.mark.parametrize("block", (32, 64, 128, 256, 512))
@pytest.mark.parametrize("P,rows,blocks", ((1, 3, 1), (2, 70, 1), (3, 5, 2), (8, 64, 21), (9, 7, 5), (16, 64, 21), (17, 3, 4), (64, 2, 10), (4, 2, 64),
                                           (2, 1100, 8)))
def test_reduced_rows_are_the_two_calls(block, P, rows, blocks):
    cols = min(block * blocks, 32768)
    partials = [_rows(p * 31 + cols, rows, cols).cuda() for p in range(P)]
    w, start = _rows(1, 1, cols)[0].cuda(), _rows(2, rows, cols).cuda()
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    eq.equarx_reduce_fused([p.view(-1) for p in partials], block, x.view(-1))
    results = []
    for reduced in (False, True):
        for residual in (None, start.clone()):
            out, packed = torch.full_like(x, 9.0), eq.alloc_mx4(rows, cols)
            codes, scales = torch.empty(rows, cols, dtype=torch.int8, device="cuda"), torch.empty(rows, cols // block, device="cuda")
            kw = dict(residual=residual, out=out, codes=codes, scales=scales, codes_block=block, mx4_codes=packed[0], mx4_scales=packed[1])
            if reduced:
                eq.equarx_norm_reduced(partials, block, w, 1e-5, **kw)
            else:
                eq.equarx_norm(x, w, 1e-5, **kw)
            results.append([t for t in (out, codes, scales, *packed, residual) if t is not None])
    for a, b in zip(results[0] + results[1], results[2] + results[3]):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("block,cols", ((32, 96), (64, 1024), (256, 5376), (512, 8192), (128, 16384)))
def test_reduced_rows_beside_strides_of_any_length(block, cols):
    """Residual and output in rows that begin on two bytes only: the bits of those that begin on sixteen."""
    rows, P = 37, 5
    partials, w = [_rows(p, rows, cols).cuda() for p in range(P)], _rows(9, 1, cols)[0].cuda()
    stream, out = _rows(8, rows, cols).cuda(), torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    wide_stream, wide_out = (torch.full((rows, cols + 3), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wide_stream[:, :cols] = stream
    eq.equarx_norm_reduced(partials, block, w, 1e-5, stream, out)
    eq.equarx_norm_reduced(partials, block, w, 1e-5, wide_stream[:, :cols], wide_out[:, :cols])
    assert torch.equal(wide_stream[:, :cols], stream) and torch.equal(wide_out[:, :cols], out)
    assert (wide_stream[:, cols:] == 9.0).all() and (wide_out[:, cols:] == 9.0).all()


def test_reduced_rows_in_place_of_a_partial():
    partials = [_rows(p, 40, 768).cuda() for p in range(5)]
    want = torch.empty_like(partials[0])
    eq.equarx_norm_reduced(partials, 128, None, out=want)
    eq.equarx_norm_reduced(partials, 128, None, out=partials[2])
    assert torch.equal(partials[2], want)


def test_a_captured_norm_replays():
    x, w, out = _rows(1, 64, 5376).cuda(), _rows(2, 1, 5376)[0].cuda(), torch.empty(64, 5376, dtype=torch.bfloat16, device="cuda")
    stream, partials = _rows(3, 64, 5376).cuda(), [_rows(4 + p, 64, 5376).cuda() for p in range(4)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eq.equarx_norm(x, w, residual=stream, out=out)
        eq.equarx_norm_reduced(partials, 128, w, residual=stream, out=out)
    for step in range(3):
        for t in (x, stream, *partials):
            t.copy_(_rows(100 + step, 64, 5376))
        expected_stream, expected = stream.clone(), torch.empty_like(out)
        graph.replay()
        torch.cuda.synchronize()
        eq.equarx_norm(x, w, residual=expected_stream, out=expected)
        eq.equarx_norm_reduced(partials, 128, w, residual=expected_stream, out=expected)
        assert torch.equal(out, expected) and torch.equal(stream, expected_stream)


def test_another_stream():
    x, out = _rows(1, 300, 1000).cuda(), torch.zeros(300, 1000, dtype=torch.bfloat16, device="cuda")
    want = torch.empty_like(out)
    eq.equarx_norm(x, None, out=want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eq.equarx_norm(x, None, out=out)
    side.synchronize()
    assert torch.equal(out, want)
