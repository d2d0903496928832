"""What the page tables' calls refuse, decided on the host before anything is launched; and their native marshalling against the checks in
Python."""
import ctypes

import pytest
import torch

import test_marshal as marshal
from paper_2506_17615_amd import binding as eq
from paper_2506_17615_amd import build
from test_serving_abi import ALIGN, NULL, OK, P, SHAPE, _refusals


@pytest.fixture(scope="module")
def lib():
    if build.is_stale():
        build.build()
    return eq.load()


def _pages(**changes):
    fields = dict(table=P[0], lengths=P[1], free=P[2], free_count=P[3], width=100, pages=1000, sequences=8, page=16)
    fields.update(changes)
    return ctypes.byref(eq._CPages(**fields))


BAD = [(SHAPE, dict(sequences=-1)), (SHAPE, dict(sequences=(1 << 20) + 1)), (SHAPE, dict(width=0)), (SHAPE, dict(width=(1 << 20) + 1)),
       (SHAPE, dict(pages=0)), (SHAPE, dict(pages=(1 << 30) + 1)), (SHAPE, dict(page=0)), (SHAPE, dict(page=-16)), (SHAPE, dict(page=65537)),
       (SHAPE, dict(pages=1 << 30, page=2048)), (NULL, dict(table=None)),
       (NULL, dict(lengths=None)), (NULL, dict(free=None)), (NULL, dict(free_count=None)), (ALIGN, dict(table=P[0] + 2)),
       (ALIGN, dict(lengths=P[1] + 1)), (ALIGN, dict(free=P[2] + 2)), (ALIGN, dict(free_count=P[3] + 2)), (SHAPE, dict(lengths=P[0] + 3196)),
       (SHAPE, dict(free=P[1])), (SHAPE, dict(free_count=P[2] + 3996))]


def test_trim_refuses(lib):
    good = dict(pages=_pages(), keep=P[4], stream=None)
    cases = [(status, dict(pages=_pages(**c))) for status, c in BAD] + [(NULL, dict(pages=None)), (SHAPE, dict(keep=P[1])),
                                                                        (SHAPE, dict(keep=P[0] + 3196)), (OK, dict(pages=_pages(sequences=0), keep=None))]
    _refusals(lib.equarx_pages_trim, good, cases, dict(keep=2))


def test_extend_refuses(lib):
    good = dict(pages=_pages(), counts=P[4], starts=P[5], slots=P[6], granted=P[7], positions=P[8], tags=P[9], row_tags=P[10], rows=64, stream=None)
    cases = [(status, dict(pages=_pages(**c))) for status, c in BAD] + [(NULL, dict(pages=None))]
    cases += [(SHAPE, c) for c in (dict(rows=-1), dict(rows=(1 << 30) + 1), dict(counts=P[5]), dict(starts=P[0]), dict(slots=P[1]),
                                   dict(granted=P[4]), dict(positions=P[6] + 508), dict(row_tags=P[9]), dict(tags=P[8]), dict(granted=P[5] + 32))]
    cases += [(NULL, dict(tags=None)), (NULL, dict(row_tags=None)), (OK, dict(pages=_pages(sequences=0), rows=0, slots=None, starts=None))]
    _refusals(lib.equarx_pages_extend, good, cases, dict(counts=2, starts=2, slots=4, granted=2, positions=2, tags=2, row_tags=2),
              optional=("granted", "positions"))


# ---------------------------------------------------------------- the binding

def _calls(device):
    pages = eq.alloc_pages(4, 6, 20, device=device)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=device)
    starts, slots, granted, positions, tags = ints(*[0] * 5), torch.zeros(20, dtype=torch.int64, device=device), ints(*[0] * 4), ints(*[0] * 20), ints(*[0] * 20)
    return {"equarx_pages_trim": ((pages, 16, ints(0, 5, 9, 1)), tuple(pages)),
            "equarx_pages_extend": ((pages, 16, ints(3, 0, 8, 5), starts, slots, granted, positions, ints(4, 3, 2, 1), tags),
                                    (*pages, starts, slots, granted, positions, tags))}


NAMES = sorted(_calls("cpu"))


def test_every_call_is_marshalled():
    assert set(NAMES) == {n for n in eq.SIGNATURES if n.startswith("equarx_pages")}


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_are_refused(name):
    eq.load()
    args, _ = _calls("cpu")[name]
    assert getattr(eq._native, name)(*args) == -1
    with pytest.raises(ValueError):
        getattr(eq, name)(*args)


@pytest.mark.parametrize("bad", (None, (), (1, 2, 3, 4), "four"))
@pytest.mark.parametrize("name", NAMES)
def test_pages_that_are_none_are_refused(name, bad):
    eq.load()
    args, _ = _calls("cpu")[name]
    with pytest.raises(ValueError):
        getattr(eq, name)(bad, *args[1:])


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
        # a replaced tensor may be a copy that the call changes: it begins both calls as it is now
        held = [t for a in changed for t in (a if isinstance(a, (list, tuple)) else [a]) if torch.is_tensor(t)]
        now = [t.clone() for t in held]
        results = []
        for f in (lambda: getattr(eq, name)(*changed), lambda: marshal._general(name, changed)):
            for o, s in zip(held + list(outputs), now + start):
                o.copy_(s)
            results.append((marshal._outcome(f), [o.clone().view(torch.uint8) for o in outputs]))
        (a, bits_a), (b, bits_b) = results
        assert a == b and all(torch.equal(p, q) for p, q in zip(bits_a, bits_b)), (name, a, b)
