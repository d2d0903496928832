"""The 4-bit and cache calls where offsets pass 32 bits."""
import pytest
import torch

from paper_2506_17615_amd import binding as eq

pytestmark = pytest.mark.gpu


def _bf16(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("new", (1, 70))
def test_a_cache_of_more_than_4_gib_is_as_a_small_one(new):
    """The same tokens in the last pages of a large pool and in a small one: the same codes, the same answers, bit by bit."""
    heads, page, dim, block = 8, 16, 256, 64
    large = (1 << 32) // (heads * page * dim) + 5000
    tokens = 330
    count = -(-tokens // page)
    small_table = torch.arange(count, dtype=torch.int32).view(1, -1).flip(1).contiguous()
    k, v, q = _bf16(1, tokens, heads, dim), _bf16(2, tokens, heads, dim), _bf16(3, new, heads * 2, dim)
    lengths, zero = torch.tensor([tokens], dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    starts = torch.tensor([0, new], dtype=torch.int32).cuda()
    answers = []
    for pages, table in ((count, small_table), (large, small_table + (large - count))):
        cache = eq.alloc_cache(pages, heads, page, dim, block)
        assert pages == count or cache.k_codes.numel() > 1 << 32
        t = torch.arange(tokens)
        slots = (table[0, t // page].long() * page + t % page).cuda()
        table = table.cuda()
        eq.equarx_cache_write(cache, k, v, slots)
        k_out, v_out, out = torch.empty_like(k), torch.empty_like(v), torch.empty_like(q)
        lse = torch.empty(new, heads * 2, device="cuda")
        eq.equarx_cache_read(cache, table, lengths, zero, k_out, v_out)
        work = eq.alloc_cache_attention_workspace(cache, new, heads * 2, 1, new, 1 << 12)
        eq.equarx_cache_attention(cache, q, starts, table, lengths, out, dim ** -0.5, new, 1 << 12, True, 0, lse, work)
        answers.append([x.clone() for x in (k_out, v_out, out, lse)] + [part[-count:].clone() for part in cache])
        # nothing else was written
        if pages != count:
            assert not any(part[:1].any() or part[pages // 2 - 500:pages // 2 + 500].any() for part in cache)
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*answers))
    assert answers[0][2].float().abs().max() > 0


def test_rows_far_from_each_other():
    """Three rows 2^31 elements apart, of x and of the output."""
    rows, cols, n, stride = 3, 300, 40, 1 << 31
    x = _bf16(4, rows, cols)
    far = torch.empty((rows - 1) * stride + cols, dtype=torch.bfloat16, device="cuda").as_strided((rows, cols), (stride, 1))
    far.copy_(x)
    packed, other = eq.alloc_mx4(rows, cols), eq.alloc_mx4(rows, cols)
    eq.equarx_mx4_quantize(x, *packed)
    eq.equarx_mx4_quantize(far, *other)
    assert all(torch.equal(a, b) for a, b in zip(packed, other))
    w = eq.alloc_mx4(n, cols)
    eq.equarx_mx4_quantize(_bf16(5, n, cols), *w)
    work = eq.alloc_mx4_workspace(rows, n, cols)
    near = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    eq.equarx_mx4_linear(x, *w, near, work)
    back = torch.empty_like(x)
    eq.equarx_mx4_dequantize(*packed, back)
    eq.equarx_mx4_dequantize(*packed, far)
    assert torch.equal(far, back)
    far.copy_(x)
    out = torch.zeros((rows - 1) * stride + n, dtype=torch.bfloat16, device="cuda").as_strided((rows, n), (stride, 1))
    eq.equarx_mx4_linear(far, *w, out, work)
    assert torch.equal(out, near)
    out.zero_()
    eq.equarx_mx4_product(*packed, *w, cols, out)
    assert torch.equal(out, near)
