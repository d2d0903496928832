"""What the 4-bit and cache calls refuse, decided on the host before anything is launched; their size queries; and their native
marshalling against the checks in Python."""
import ctypes

import pytest
import torch

import test_marshal as marshal
from paper_2506_17615_amd import binding as eq
from paper_2506_17615_amd import build

A = 0x7F0000000000          # never dereferenced, 1 GiB apart from each other
P = [A + (i << 30) for i in range(12)]
OK, NULL, SHAPE, BLOCK, ALIGN, SMALL = (eq.STATUS_OK, eq.STATUS_NULL_POINTER, eq.STATUS_BAD_SHAPE, eq.STATUS_BAD_BLOCK,
                                        eq.STATUS_MISALIGNED, eq.STATUS_WORKSPACE_TOO_SMALL)


@pytest.fixture(scope="module")
def lib():
    if build.is_stale():
        build.build()
    return eq.load()


def _refusals(call, good, cases, pointers, optional=()):
    """Every case is `good` with some arguments replaced; every pointer is refused as NULL (but the optional) and off its alignment."""
    names = list(good)

    def with_(**changes):
        return call(*[changes.get(n, good[n]) for n in names])

    for name, offset in pointers.items():
        if name not in optional:
            assert with_(**{name: None}) == NULL, name
        assert with_(**{name: good[name] + offset}) == ALIGN, name
    for status, changes in cases:
        assert with_(**changes) == status, (status, changes)


def test_mx4_sizes(lib):
    assert [eq.mx4_row_blocks(n) for n in (0, 1, 128, 129, 5376)] == [0, 4, 4, 8, 168]
    assert lib.equarx_mx4_row_blocks(-1) == 0 and lib.equarx_mx4_row_blocks(1 << 31) == 0
    size = lib.equarx_mx4_workspace_bytes
    assert size(4096, 64, 300) == 4096 * 192 + 4096 * 12 and size(1, 64, 300) == 0
    assert size(0, 4, 4) == 0 and size(-1, 4, 4) == 0 and size(4, 4, (1 << 24) + 1) == 0


def test_mx4_rows_refuse(lib):
    good = dict(x=P[0], rows=8, cols=200, stride=200, codes=P[1], scales=P[2], stream=None)
    shapes = [(SHAPE, c) for c in (dict(rows=-1), dict(cols=-1), dict(stride=199), dict(rows=1 << 31), dict(cols=1 << 31, stride=1 << 31),
                                   dict(rows=1 << 30, cols=1 << 11, stride=1 << 11))]
    nothing = [(OK, dict(rows=0, x=None, codes=None, scales=None)), (OK, dict(cols=0, stride=0, x=None, codes=None, scales=None))]
    overlaps = [(SHAPE, c) for c in (dict(codes=P[0]), dict(codes=P[0] + 16), dict(scales=P[0] + 8 * 400 - 16), dict(scales=P[1] + 16),
                                     dict(codes=P[2] - 16))]
    pointers = dict(x=8, codes=4, scales=2)
    _refusals(lib.equarx_mx4_quantize, good, shapes + nothing + overlaps, pointers)
    back = dict(codes=P[1], scales=P[2], rows=8, cols=200, out=P[0], stride=200, stream=None)
    _refusals(lib.equarx_mx4_dequantize, back, shapes + [(SHAPE, dict(out=P[1])), (SHAPE, dict(out=P[2] - 16)), (OK, dict(rows=0, out=None))],
              dict(out=8, codes=4, scales=2))


def test_mx4_products_refuse(lib):
    M, N, K = 70, 96, 300
    need = lib.equarx_mx4_workspace_bytes(M, N, K)
    shapes = [(SHAPE, c) for c in (dict(M=-1), dict(N=-1), dict(K=-1), dict(out_stride=95), dict(K=(1 << 24) + 1), dict(M=1 << 31),
                                   dict(N=1 << 31, out_stride=1 << 31))]
    tail = dict(M=M, N=N, K=K, out=P[4], out_stride=N, workspace=P[5], nbytes=need, stream=None)
    over = [(SHAPE, c) for c in (dict(out=P[2]), dict(out=P[3] - 16), dict(out=P[0] + 16))]
    good = dict(xc=P[0], xs=P[1], wc=P[2], ws=P[3], **tail)
    pointers = dict(xc=4, xs=4, wc=4, ws=4, out=8)
    _refusals(lib.equarx_mx4_product, good, shapes + over + [(OK, dict(M=0, out=None))], pointers)
    good = dict(x=P[0], stride=K, wc=P[2], ws=P[3], **tail)
    cases = shapes + over + [(SHAPE, dict(stride=K - 1)), (SMALL, dict(nbytes=need - 1)), (SHAPE, dict(workspace=P[4])),
                             (SHAPE, dict(workspace=P[0] - 256)), (SHAPE, dict(workspace=P[2])), (OK, dict(N=0, out=None))]
    _refusals(lib.equarx_mx4_linear, good, cases, dict(x=8, wc=4, ws=4, out=8, workspace=16))


def _cache(**changes):
    fields = dict(k_codes=P[0], k_scales=P[1], v_codes=P[2], v_scales=P[3], pages=10, heads=2, page=16, dim=128, block=64)
    fields.update(changes)
    return ctypes.byref(eq._CCache(**fields))


BAD_CACHES = [(SHAPE, dict(dim=96)), (SHAPE, dict(dim=0)), (BLOCK, dict(block=32)), (BLOCK, dict(block=256)), (BLOCK, dict(block=0)),
              (SHAPE, dict(page=8)), (SHAPE, dict(page=24)), (SHAPE, dict(page=0)), (SHAPE, dict(page=65552)), (SHAPE, dict(pages=0)),
              (SHAPE, dict(pages=-1)), (SHAPE, dict(pages=1 << 31)), (SHAPE, dict(heads=0)), (SHAPE, dict(heads=65536)),
              (SHAPE, dict(pages=1 << 30, heads=8)), (NULL, dict(k_codes=None)), (NULL, dict(v_scales=None)),
              (ALIGN, dict(v_codes=P[2] + 8)), (ALIGN, dict(k_scales=P[1] + 4))]


def _cache_cases(cases):
    return [(status, dict(cache=_cache(**c))) for status, c in BAD_CACHES] + [(NULL, dict(cache=None))] + cases


def test_cache_write_refuses(lib):
    good = dict(cache=_cache(), k=P[4], k_row=256, k_head=128, v=P[5], v_row=256, v_head=128, tokens=30, slots=P[6], stream=None)
    cases = [(SHAPE, dict(tokens=-1)), (SHAPE, dict(tokens=(1 << 30) + 1)), (ALIGN, dict(k_row=260)), (ALIGN, dict(v_head=129)),
             (SHAPE, dict(k_row=-256)), (SHAPE, dict(v_row=1 << 40)), (SHAPE, dict(v_head=1 << 41)), (SHAPE, dict(k=P[0] + 64)),
             (SHAPE, dict(v=P[3] - 64)), (SHAPE, dict(slots=P[1])), (SHAPE, dict(cache=_cache(k_scales=P[0] + 64))),
             (SHAPE, dict(cache=_cache(v_codes=P[0]))), (OK, dict(tokens=0, k=None, v=None, slots=None))]
    _refusals(lib.equarx_cache_write, good, _cache_cases(cases), dict(k=8, v=2, slots=4))


def test_cache_read_refuses(lib):
    good = dict(cache=_cache(), table=P[4], width=3, lengths=P[5], starts=P[6], sequences=4, longest=48, rows=100, k=P[7], v=P[8], stream=None)
    cases = [(SHAPE, c) for c in (dict(width=-1), dict(width=1 << 31), dict(sequences=-1), dict(longest=-1), dict(rows=-1), dict(rows=1 << 31),
                                  dict(k=P[8]), dict(k=P[0]), dict(v=P[4] - 64), dict(v=P[3] - 64), dict(k=P[8] + 64))]
    cases += [(OK, dict(sequences=0, table=None, lengths=None, k=None)), (OK, dict(rows=0, k=None, v=None))]
    _refusals(lib.equarx_cache_read, good, _cache_cases(cases), dict(table=2, lengths=2, starts=2, k=8, v=8))


def test_cache_attention_refuses(lib):
    size = lib.equarx_cache_attention_workspace_bytes
    need = size(2, 128, 20, 8, 4, 1, 5000)
    assert need > 0 and size(2, 128, 20, 8, 4, 1, 500) == 0 and size(2, 128, 20, 7, 4, 1, 500) == 0 and size(2, 96, 20, 8, 4, 1, 5000) == 0
    good = dict(cache=_cache(), q=P[4], q_rows=20, q_heads=8, q_row=1024, q_head=128, starts=P[5], table=P[6], width=400, lengths=P[7],
                sequences=4, scale=0.1, queries=1, longest=5000, flags=1, window=0, out=P[8], lse=P[9], workspace=P[10], nbytes=need,
                stream=None)
    cases = [(SHAPE, c) for c in (dict(q_rows=-1), dict(q_rows=1 << 28), dict(q_heads=0), dict(q_heads=7), dict(q_row=-8), dict(q_row=1 << 40),
                                  dict(sequences=-1), dict(width=0), dict(width=1 << 31), dict(queries=0), dict(longest=0),
                                  dict(longest=(1 << 31) - 1), dict(flags=2), dict(flags=3), dict(window=-1), dict(flags=0, window=5),
                                  dict(out=P[4]), dict(out=P[0]), dict(out=P[4] + 20 * 2048 - 16), dict(lse=P[8]), dict(lse=P[5]),
                                  dict(workspace=P[8]), dict(workspace=P[2]), dict(workspace=P[6]))]
    cases += [(ALIGN, dict(q_row=1028)), (ALIGN, dict(q_head=130)), (SMALL, dict(nbytes=need - 1)), (SMALL, dict(nbytes=0)),
              (OK, dict(sequences=0, q=None, out=None)), (OK, dict(q_rows=0, q=None, out=None))]
    _refusals(lib.equarx_cache_attention, good, _cache_cases(cases),
              dict(q=8, starts=2, table=2, lengths=2, out=8, lse=8, workspace=128), optional=("lse",))


# ---------------------------------------------------------------- the binding

def _calls(device):
    gen = torch.Generator().manual_seed(6)

    def bf16(*shape):
        return torch.randn(*shape, generator=gen).to(torch.bfloat16).to(device)

    def ints(values, dtype=torch.int32):
        return torch.tensor(values, dtype=dtype, device=device)

    M, N, K = 40, 48, 200
    x, w, out = bf16(M, K), bf16(N, K), bf16(M, N)
    packed = [torch.randint(0, 120, (r, 8 * n), generator=gen).to(torch.uint8).to(device) for r in (M, N) for n in (16, 1)]
    px, pw = packed[:2], packed[2:]
    work = torch.zeros(1 << 22, dtype=torch.uint8, device=device)
    cache = eq.alloc_cache(9, 2, 16, 64, 64, device=device)
    for codes, scales in (cache[:2], cache[2:]):
        codes.copy_(torch.randint(-127, 128, codes.shape, generator=gen))
        scales.copy_(torch.rand(scales.shape, generator=gen))
    table, lengths = ints([[0, 3, 5], [7, 1, 2]]), ints([40, 33])
    k, v, slots = bf16(16, 2, 64), bf16(16, 2, 64), ints([5 + 3 * i for i in range(16)], torch.int64)
    k_out, v_out = bf16(80, 2, 64), bf16(80, 2, 64)
    q, attended, lse = bf16(24, 8, 64), bf16(24, 8, 64), torch.zeros(24, 8, device=device)
    return {
        "equarx_mx4_quantize": ((x, *px), tuple(px)),
        "equarx_mx4_dequantize": ((*px, x), (x,)),
        "equarx_mx4_product": ((*px, *pw, K, out, work), (out,)),
        "equarx_mx4_linear": ((x, *pw, out, work), (out,)),
        "equarx_cache_write": ((cache, k, v, slots), tuple(cache)),
        "equarx_cache_read": ((cache, table, lengths, ints([0, 40]), k_out, v_out, 40), (k_out, v_out)),
        "equarx_cache_attention": ((cache, q, ints([0, 9, 24]), table, lengths, attended, 0.125, 15, 40, True, 17, lse, work), (attended, lse)),
    }


NAMES = sorted(_calls("cpu"))


def test_every_serving_call_is_marshalled():
    assert set(NAMES) == {n for n in eq.SIGNATURES if n.startswith(("equarx_mx4", "equarx_cache")) and "bytes" not in n and "blocks" not in n}


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_are_refused(name):
    eq.load()
    args, _ = _calls("cpu")[name]
    assert getattr(eq._native, name)(*args) == -1
    with pytest.raises(ValueError):
        getattr(eq, name)(*args)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_the_native_path_and_the_general_one_agree(name):
    """The plain call is taken natively; and any other ends the same way on both paths: the same exception, or the same bits."""
    eq.load()
    args, outputs = _calls("cuda")[name]
    start = [o.clone() for o in outputs]
    assert getattr(eq._native, name)(*args) == 0
    for changed in [args] + list(marshal._altered(args)):
        if any(hasattr(a, "__next__") for a in changed):        # can be gone through once
            continue
        results = []
        for f in (lambda: getattr(eq, name)(*changed), lambda: marshal._general(name, changed)):
            for o, s in zip(outputs, start):
                o.copy_(s)
            results.append((marshal._outcome(f), [o.clone().view(torch.uint8) for o in outputs]))
        (a, bits_a), (b, bits_b) = results
        assert a == b and all(torch.equal(p, q) for p, q in zip(bits_a, bits_b)), (name, a, b)
