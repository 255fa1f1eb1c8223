"""sss_kv_store_q4 of 16-bit values at and beside every tie: for each significand of a group's
largest value, what lies next to the quotients' half-integers on either side, equal to the oracle's
quantizer (which divides exactly) to the last bit."""
import numpy as np
import pytest
import torch

from paper_2607_08779_gb300 import sss
from test_gpu_kv_q4 import DEV, expect, filled, ints

pytestmark = pytest.mark.gpu


def beside_ties(top, dtype):
    """31 values of the type around top (2 n + 1) / 16, n = 0 .. 7: the nearest below and above, and
    the tie itself where the type has it; signs alternate."""
    ties = top * (2 * np.arange(8) + 1) / 16  # exact in 64 bits
    near = torch.from_numpy(ties).to(dtype)   # rounded to nearest
    out = [near.double().numpy()]
    bits = near.view(torch.int16)
    for step in (1, -1):
        out.append((bits + step).view(dtype).double().numpy())
    v = np.concatenate(out)                   # 24 values, each tie enclosed
    v = np.concatenate([v, -v[:7]])
    v[1::2] *= -1
    return np.clip(v, -top, top)


@pytest.mark.parametrize("dtype,bits,exponent", [(torch.float16, 11, e) for e in (0, 4, -9, -12)] +
                         [(torch.bfloat16, 8, e) for e in (0, 7, -9, 100, -100, -118)])
def test_every_significand(dtype, bits, exponent):
    rows = []
    for b in range(1 << (bits - 1), 1 << bits):
        top = b * 2.0 ** (exponent - bits + 1)
        around = beside_ties(top, dtype)
        rows.append(np.concatenate([[top], around, [-top], np.where(np.abs(around) == top, around / 2, around)]))
    x = torch.from_numpy(np.array(rows)).to(dtype)
    assert torch.equal(x.double(), torch.from_numpy(np.array(rows)))  # (all are of the type)
    x = x.view(-1, 1, 64)
    n = x.shape[0]
    c, status = filled(-(-n // 256), 256, 1, 64), ints([0])
    sss.sss_kv_store_q4(x.to(DEV), x.to(DEV), c, dev_status=status)
    assert np.array_equal(c.blocks.cpu().numpy(), expect(x, x, list(range(n)), c))
    got, _ = sss.sss_kv_fetch_q4(c, ints(list(range(n))))
    assert bool(torch.isfinite(got).all())
