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


def test_an_error_names_what_a_serving_call_may_have_wrong():
    """Not the reduction's arguments and queries alone: these statuses come from every call."""
    text = {s: eq.status_string(s) for s in (eq.STATUS_BAD_SHAPE, eq.STATUS_BAD_BLOCK, eq.STATUS_MISALIGNED, eq.STATUS_WORKSPACE_TOO_SMALL)}
    assert "stride" in text[eq.STATUS_BAD_SHAPE] and "stride" in text[eq.STATUS_MISALIGNED] and "cache" in text[eq.STATUS_BAD_BLOCK]
    assert "the call's equarx_..._workspace_bytes()" in text[eq.STATUS_WORKSPACE_TOO_SMALL]
