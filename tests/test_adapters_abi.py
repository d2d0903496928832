"""What a call of adapters refuses, decided on the host before anything is launched; its workspace; and its native marshalling against the
checks in Python."""
import ctypes

import pytest
import torch

import test_marshal as marshal
from paper_2506_17615_amd import binding as eq
from paper_2506_17615_amd import build
from test_serving_abi import ALIGN, NULL, OK, P, SHAPE, SMALL, _refusals


@pytest.fixture(scope="module")
def lib():
    if build.is_stale():
        build.build()
    return eq.load()


def test_workspace(lib):
    size = lib.equarx_adapters_workspace_bytes
    assert size(64, 512, 300, 16, 3, 32) > 0
    for nothing in ((0, 4, 4, 8, 1, 1), (4, 0, 4, 8, 1, 1), (4, 4, 0, 8, 1, 1), (-1, 4, 4, 8, 1, 1), (4, 4, 4, 7, 1, 1), (4, 4, 4, 0, 1, 1),
                    (4, 4, 4, 136, 1, 1), (4, 4, 4, 8, 0, 1), (4, 4, 4, 8, 5, 1), (4, 4, 4, 8, 1, 0), (4, 4, 4, 8, 1, 8193),
                    ((1 << 24) + 1, 4, 4, 8, 1, 1), (4, (1 << 22) + 1, 4, 8, 1, 1), (4, 4, (1 << 22) + 1, 8, 1, 1)):
        assert size(*nothing) == 0, nothing
    for most in ((1 << 24, 1 << 22, 1 << 22, 128, 1, 1), (1, 1 << 22, 8, 8, 1, 8192), (1 << 24, 64, 64, 8, 4, 8192)):
        assert size(*most) > 0


def _ends(*columns):
    return (ctypes.c_int64 * len(columns))(*columns)


def test_adapters_refuse(lib):
    M, N, K = 70, 300, 200
    need = lib.equarx_adapters_workspace_bytes(M, N, K, 16, 2, 5)
    good = dict(x=P[0], x_stride=K, a=P[1], b=P[2], factors=P[3], adapters=5, rank=16, ids=P[4], M=M, N=N, K=K, ends=_ends(100, 300), slices=2,
                out=P[5], out_stride=N, workspace=P[6], nbytes=need, stream=None)
    cases = [(SHAPE, c) for c in (dict(M=-1), dict(N=-1), dict(K=-1), dict(M=(1 << 24) + 1), dict(N=(1 << 22) + 1), dict(K=(1 << 22) + 1),
                                  dict(rank=0), dict(rank=-8), dict(rank=12), dict(rank=136), dict(slices=0), dict(slices=5), dict(adapters=0),
                                  dict(adapters=8193), dict(x_stride=K - 1), dict(out_stride=N - 1), dict(x_stride=1 << 40), dict(out_stride=1 << 40),
                                  dict(ends=_ends(100, 299)), dict(ends=_ends(301, 300)), dict(ends=_ends(-1, 300)), dict(ends=_ends(300, 100)),
                                  dict(out=P[0]), dict(out=P[2] + 16), dict(out=P[3]), dict(out=P[4]), dict(workspace=P[5]), dict(workspace=P[1]),
                                  dict(workspace=P[0] + 512))]
    cases += [(NULL, dict(ends=None)), (SMALL, dict(nbytes=need - 1)), (OK, dict(M=0, x=None, out=None)), (OK, dict(N=0, ends=_ends(0, 0), out=None)),
              (OK, dict(K=0, x=None, a=None, workspace=None, nbytes=0))]
    _refusals(lib.equarx_adapters, good, cases, dict(x=8, a=8, b=8, factors=2, ids=2, out=8, workspace=16))


# ---------------------------------------------------------------- the binding

def _calls(device):
    gen = torch.Generator().manual_seed(8)
    bf16 = lambda *shape: torch.randn(*shape, generator=gen).to(torch.bfloat16).to(device)
    out = bf16(20, 96)
    return {"equarx_adapters": ((bf16(20, 40), bf16(3, 16, 40), bf16(3, 96, 8), torch.rand(3, generator=gen).to(device),
                                 torch.randint(-1, 4, (20,), generator=gen).to(torch.int32).to(device), out, (32, 96),
                                 torch.zeros(1 << 20, dtype=torch.uint8, device=device)), (out,))}


NAMES = sorted(_calls("cpu"))


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
    slices = [args[:6] + (ends, args[7]) for ends in (None, (96,), (96.0,), (40, 96), (97,), (95,), (0, 96), (50, 40), [32, 96], (1, 2, 3, 4, 96), (), "96")]
    altered = [tuple(c[:6]) + args[6:7] + tuple(c[6:]) for c in marshal._altered(args[:6] + args[7:])]      # of all that are tensors
    for changed in [args] + slices + altered:
        if any(hasattr(a, "__next__") for a in changed):        # can be gone through once
            continue
        results = []
        for f in (lambda: getattr(eq, name)(*changed), lambda: marshal._general(name, changed)):
            for o, s in zip(outputs, start):
                o.copy_(s)
            results.append((marshal._outcome(f), [o.clone().view(torch.uint8) for o in outputs]))
        (a, bits_a), (b, bits_b) = results
        assert a == b and all(torch.equal(p, q) for p, q in zip(bits_a, bits_b)), (name, a, b)
