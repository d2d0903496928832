"""What extending the page tables refuses of the lengths that attention sees, decided on the host before anything is launched."""
import ctypes

import pytest
import torch

from paper_2506_17615_amd import binding as eq
from test_pages_abi import NAMES, _calls, _pages, lib                    # noqa: F401  (lib: the fixture)
from test_serving_abi import ALIGN, OK, P, SHAPE


@pytest.mark.parametrize("status,seen", ((ALIGN, P[11] + 2), (SHAPE, P[0] + 3196), (SHAPE, P[1]), (SHAPE, P[2]), (SHAPE, P[3]), (SHAPE, P[4]),
                                         (SHAPE, P[5] + 32), (SHAPE, P[6] + 508), (SHAPE, P[7]), (SHAPE, P[8]), (SHAPE, P[9]), (SHAPE, P[10] + 252)))
def test_extend_refuses(lib, status, seen):                              # noqa: F811
    assert lib.equarx_pages_extend(_pages(seen=seen), *P[4:11], 64, None) == status


def test_without_sequences_nothing_is_seen(lib):                         # noqa: F811
    assert lib.equarx_pages_extend(_pages(sequences=0, seen=None), None, None, None, None, None, None, None, 0, None) == OK


def test_the_structure_is_the_headers():
    """Fields by their offsets: what was there is where it was."""
    offsets = [getattr(eq._CPages, name).offset for name, _ in eq._CPages._fields_]
    assert offsets == [0, 8, 16, 24, 32, 40, 48, 52, 56] and ctypes.sizeof(eq._CPages) == 64


def test_the_binding_refuses():
    eq.load()
    args, _ = _calls("cpu")["equarx_pages_extend"]
    for seen in (None, torch.zeros(4, dtype=torch.int32), 5):
        assert eq._native.equarx_pages_extend(*args, seen) == -1
        with pytest.raises(ValueError):
            eq.equarx_pages_extend(*args, seen)


@pytest.mark.gpu
def test_the_native_path_and_the_general_one_agree():
    import test_marshal as marshal
    eq.load()
    args, outputs = _calls("cuda")["equarx_pages_extend"]
    seen = torch.full((4,), 9, dtype=torch.int32, device="cuda")
    start = [o.clone() for o in outputs]
    for last in (seen, None, seen[:3], seen.long(), seen.cpu(), torch.zeros(8, dtype=torch.int32, device="cuda")[::2], args[0][1]):
        results = []
        for f in (lambda: eq.equarx_pages_extend(*args, last), lambda: marshal._general("equarx_pages_extend", (*args, last))):
            for o, s in zip(outputs, start):
                o.copy_(s)
            seen.fill_(9)
            results.append((marshal._outcome(f), [o.clone() for o in (*outputs, seen)]))
        (a, bits_a), (b, bits_b) = results
        assert a == b and all(torch.equal(p, q) for p, q in zip(bits_a, bits_b))
        assert (a[1] is None) == (last is None or last is seen)
