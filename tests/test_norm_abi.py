"""What the norms refuse, decided on the host before anything is launched; and their native marshalling against the checks in Python."""
import ctypes

import pytest
import torch

import test_marshal as marshal
from paper_2506_17615_amd import binding as eq
from paper_2506_17615_amd import build
from test_serving_abi import ALIGN, BLOCK, NULL, OK, P, SHAPE, _refusals


@pytest.fixture(scope="module")
def lib():
    if build.is_stale():
        build.build()
    return eq.load()


def _outputs(**changes):
    fields = dict(out_bf16=P[4], out_stride=256, codes=P[5], scales=P[6], mx4_codes=P[7], mx4_scales=P[8], block=128)
    fields.update(changes)
    return ctypes.byref(eq._CNormOutputs(**fields))


NONE = dict(out_bf16=None, codes=None, scales=None, mx4_codes=None, mx4_scales=None)
OUTPUTS = [(NULL, NONE), (NULL, dict(codes=None)), (NULL, dict(scales=None)), (NULL, dict(mx4_codes=None)), (NULL, dict(mx4_scales=None)),
           (BLOCK, dict(block=0)), (BLOCK, dict(block=48)), (BLOCK, dict(block=1024)), (SHAPE, dict(block=512)), (SHAPE, dict(out_stride=255)),
           (SHAPE, dict(out_stride=1 << 40)), (ALIGN, dict(out_bf16=P[4] + 8)), (ALIGN, dict(codes=P[5] + 4)), (ALIGN, dict(scales=P[6] + 4)),
           (ALIGN, dict(mx4_codes=P[7] + 4)), (ALIGN, dict(mx4_scales=P[8] + 4)), (SHAPE, dict(codes=P[4])), (SHAPE, dict(out_bf16=P[1])),
           (SHAPE, dict(scales=P[5] + 16)), (SHAPE, dict(mx4_codes=P[1] + 16)), (SHAPE, dict(mx4_scales=P[0])), (SHAPE, dict(out_bf16=P[0] + 16)),
           (SHAPE, dict(out_bf16=P[2]))]


def _cases():
    cases = [(status, dict(outputs=_outputs(**c))) for status, c in OUTPUTS] + [(NULL, dict(outputs=None))]
    cases += [(SHAPE, c) for c in (dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(cols=32768 + 1), dict(cols=1 << 31),
                                   dict(residual_stride=255), dict(residual_stride=1 << 40), dict(eps=-1e-9), dict(eps=float("nan")),
                                   dict(eps=float("inf")), dict(flags=2), dict(flags=3), dict(flags=1, weight=None), dict(residual=P[2]))]
    return cases + [(OK, dict(rows=0, outputs=None)), (OK, dict(cols=0, outputs=None))]


COMMON = dict(residual=P[1], residual_stride=256, weight=P[2], rows=20, cols=256, eps=1e-6, flags=0)


def test_norm_refuses(lib):
    good = dict(x=P[0], x_stride=256, **COMMON, outputs=_outputs(), stream=None)
    cases = _cases() + [(SHAPE, dict(x_stride=255)), (SHAPE, dict(x_stride=1 << 40)), (SHAPE, dict(x=P[1])), (SHAPE, dict(x=P[1] + 16)),
                        (SHAPE, dict(x_stride=257, outputs=_outputs(out_bf16=P[0])))]
    _refusals(lib.equarx_norm, good, cases, dict(x=8, residual=8, weight=2), optional=("residual", "weight"))


def test_norm_of_a_reduction_refuses(lib):
    table = lambda *a: (ctypes.c_void_p * len(a))(*a)
    good = dict(partials=table(P[0], P[3]), P=2, block=64, **COMMON, outputs=_outputs(), stream=None)
    cases = _cases() + [(NULL, dict(partials=table(P[0], None))), (ALIGN, dict(partials=table(P[0] + 8, P[3]))), (SHAPE, dict(P=0)),
                        (SHAPE, dict(P=65)), (BLOCK, dict(block=0)), (BLOCK, dict(block=96)), (SHAPE, dict(block=512)), (SHAPE, dict(cols=255)),
                        (SHAPE, dict(partials=table(P[0], P[1]))), (SHAPE, dict(outputs=_outputs(out_bf16=P[3], out_stride=257))),
                        (NULL, dict(partials=None))]
    _refusals(lib.equarx_norm_reduced, good, cases, dict(residual=8, weight=2), optional=("residual", "weight"))


# ---------------------------------------------------------------- the binding

def _calls(device):
    gen = torch.Generator().manual_seed(7)
    bf16 = lambda *shape: torch.randn(*shape, generator=gen).to(torch.bfloat16).to(device)
    rows, cols = 12, 256
    codes, scales = torch.zeros(rows, cols, dtype=torch.int8, device=device), torch.zeros(rows, cols // 64, device=device)
    packed = [torch.zeros(rows, n, dtype=torch.uint8, device=device) for n in (128, 8)]
    residual, out = bf16(rows, cols), bf16(rows, cols)
    tail = (bf16(cols), 1e-6, residual, out, codes, scales, 64, *packed, True)
    outputs = (residual, out, codes, scales, *packed)
    return {"equarx_norm": ((bf16(rows, cols), *tail), outputs),
            "equarx_norm_reduced": (([bf16(rows, cols) for _ in range(3)], 64, *tail), outputs)}


NAMES = sorted(_calls("cpu"))


def test_every_norm_is_marshalled():
    assert set(NAMES) == {n for n in eq.SIGNATURES if n.startswith("equarx_norm")}


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


def test_a_tensor_of_another_device_is_refused(monkeypatch):
    """The call would be made on the current device's stream."""
    class On:
        def __init__(self, index):
            self.device = torch.device("cuda", index)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    eq._need_here(None, On(0))
    with pytest.raises(ValueError, match="current device"):
        eq._need_here(On(0), On(1))
