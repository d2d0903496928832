"""The serving calls' defaults in the binding, on the host."""
import pytest
import torch

from paper_2506_17615_amd import binding as eq


def _reading():
    cache = eq.alloc_cache(2, 1, 16, 64, 64, device="cpu")
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    out = torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    return dict(cache=cache, page_table=ints(1, 2), lengths=ints(1), starts=ints(1), k_out=out, v_out=out.clone())


@pytest.mark.parametrize("name,bad", [(n, None) for n in _reading()] + [("cache", ()), ("cache", (1, 2, 3, 4)), ("cache", "four"),
                                                                        ("page_table", 3), ("page_table", torch.zeros((), dtype=torch.int32))])
def test_reading_back_without_a_length_is_refused_like_any_call(name, bad):
    eq.load()
    args = _reading()
    args[name] = bad
    with pytest.raises(ValueError):
        eq.equarx_cache_read(**args)
    with pytest.raises(ValueError):
        eq.equarx_cache_read(**args, max_length=16)
