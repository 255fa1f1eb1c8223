"""sss_attention over a cache without slots, of more tokens than one dimension of a grid has
tiles for: zeros."""
import pytest
import torch

from paper_2607_08779_gb300 import sss

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("kv", [0, 3])
def test_a_long_prompt_over_a_cache_without_slots(kv):
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    q = torch.randn((300000, 8, 64), device=DEV).bfloat16()
    none = torch.zeros((0, 1, 64), dtype=torch.bfloat16, device=DEV)
    status = ints([0])
    out = torch.full_like(q, 7.0)
    sss.sss_attention(q, sss.KVCache(none, none, 16), ints([0, 300000]), ints([kv]), 300000, kv, block_table=ints([[0]]),
                      out=out, dev_status=status)
    assert int(status) == (sss.FLAG_INDEX if kv else 0) and not out.any()
