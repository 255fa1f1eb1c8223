"""sss_attention_q4 of few rows in more tiles than one dimension of a grid holds (65535)."""
import numpy as np
import pytest
import torch

from paper_2607_08779_gb300 import sss
from test_gpu_attention_q4 import BF, DEV, make, cache_of

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("batch,fresh,hq", [(16384, 8, 8), (65535, 5, 12)])
def test_drafted_tokens_of_many_requests(batch, fresh, hq):
    # requests of a few keys, in the same pages over and over; some without tokens
    few = make([fresh] * 40, [fresh + 3 * i % 60 for i in range(40)], hq, 1, 64, BF, 16, seed=95)
    of = np.random.default_rng(1).integers(0, 40, batch)
    n = np.where(np.arange(batch) % 97 == 5, 0, fresh)
    cu = np.concatenate([[0], np.cumsum(n)])
    q = few["q"].to(DEV).view(40, fresh, hq, 64)[torch.as_tensor(of[n > 0], device=DEV)].reshape(-1, hq, 64)
    table, kv = ints(few["table"].numpy()[of]), ints(np.asarray(few["kv"])[of])
    status = ints([0])
    cache = cache_of(few)
    got = sss.sss_attention_q4(q, cache, ints(cu), kv, fresh, max(few["kv"]), table, dev_status=status)
    want = sss.sss_attention_q4(few["q"].to(DEV), cache, ints(few["cu"]), ints(few["kv"]), fresh, max(few["kv"]),
                                few["table"].to(DEV), dev_status=status)
    again = want.view(40, fresh, hq, 64)[torch.as_tensor(of[n > 0], device=DEV)].reshape(-1, hq, 64)
    assert int(status) == 0
    # (a few requests are split over CTAs otherwise: within what p and the sums are rounded by, and the output)
    assert float((got.float() - again.float()).abs().max()) <= 2 * 2.0 ** -8 * float(again.float().abs().max())


def test_a_long_prompt_without_keys():
    # no keys: zeros, however many tokens
    q = torch.randn((200000, 8, 64), device=DEV).to(BF)
    cache, status = sss.empty_kv_cache_q4(2, 16, 1, 64), ints([0])
    out = torch.full(q.shape, 7.0, dtype=BF, device=DEV)
    sss.sss_attention_q4(q, cache, ints([0, 200000]), ints([0]), 200000, 0, ints([[0]]), out=out, dev_status=status)
    assert int(status) == 0 and not out.any()
