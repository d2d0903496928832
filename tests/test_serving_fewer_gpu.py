"""A layer made for many sequences, called with fewer."""
import pytest
import torch

from paper_2506_17615_amd import serving
from test_serving_layer_gpu import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prompts,hint", (([300], 300), ([128], 128), ([100, 3], 100), ([60, 60, 60, 60], 60), ([200], 3), ([1], 1)))
def test_fewer_sequences_than_the_layer_was_made_for(prompts, hint):
    """One prompt alone is cut into splits where 300 sequences are not; `hint`: what the caller says is the longest run."""
    heads, kv_heads, dim, hidden, page, width = 8, 2, 64, 192, 16, 32
    gen = torch.Generator().manual_seed(11)
    bf16 = lambda *shape: torch.randn(*shape, generator=gen).mul_(shape[-1] ** -0.5).to(torch.bfloat16).cuda()
    layer = serving.ShardedAttention(bf16((heads + 2 * kv_heads) * dim, hidden), bf16(hidden, heads * dim), 1, heads, kv_heads, dim,
                                     4 * width, page, 300, 300, 512)
    tokens, count = sum(prompts), len(prompts)
    table = torch.randperm(count * width, generator=gen).to(torch.int32).view(count, width)
    starts = [0, *torch.tensor(prompts).cumsum(0).tolist()]
    x, out = bf16(tokens, hidden) * 10, torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda")
    on = lambda values: torch.tensor(values, dtype=torch.int32).cuda()
    layer(x, serving.slots_of(table, page, prompts, prompts).cuda(), on(starts), table.cuda(), on(prompts), hint, out)
    _check(layer, x, starts, table, prompts, out, page)
