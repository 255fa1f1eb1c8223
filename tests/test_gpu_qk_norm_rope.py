"""sss_qk_norm_rope against a plain 64-bit form, within the bound that
attn_plain.norm_rope_bound derives from its roundings."""
import numpy as np
import pytest
import torch

import attn_plain
from paper_2607_08779_gb300 import sss

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32


def make(t, hq, hkv, dim, in_dtype=F32, dtype=BF, norm=(True, True), half=True, rot=None, fused=False,
         page=16, seed=0, most=500):
    g = torch.Generator().manual_seed(seed)
    rot = dim if rot is None else rot
    widths = [hq * dim, hkv * dim, hkv * dim]
    x = torch.randn((t, sum(widths) + 8), generator=g).to(in_dtype).to(DEV)
    q, k, v = x[:, 8:].split(widths, dim=1) if fused else (p.contiguous() for p in x[:, 8:].split(widths, dim=1))
    slots = -(-t // page) * page + 2 * page
    c = dict(q=q, k=k, v=v, dim=dim, rot=rot, half=half, dtype=dtype, eps=1e-5)
    c["wq"], c["wk"] = ((1 + 0.3 * torch.randn((dim,), generator=g)).to(DEV) if n else None for n in norm)
    c["cos"], c["sin"] = (torch.rand((most, rot // 2), generator=g).mul(2).sub(1).to(DEV) for _ in range(2))
    c["positions"] = torch.randint(0, most, (t,), generator=g).int().to(DEV)
    c["slots"] = torch.randperm(slots, generator=g)[:t].int().to(DEV)
    c["kc"], c["vc"] = (torch.randn((slots, hkv, dim), generator=g).to(dtype).to(DEV) for _ in range(2))
    return c


def call(c, status=None, slots="own", positions="own", **kw):
    rope = sss.Rope(c["cos"] if c["rot"] else None, c["sin"] if c["rot"] else None,
                    sss.ROPE_HALF if c["half"] else sss.ROPE_PAIRS, c["wq"], c["wk"], c["eps"])
    kc, vc = c["kc"].clone(), c["vc"].clone()
    out = sss.sss_qk_norm_rope(c["q"], c["k"], c["v"], rope, c["positions"] if positions == "own" else positions,
                               sss.KVCache(kc, vc, 16), slots=c["slots"] if slots == "own" else slots,
                               dev_status=status, **kw)
    torch.cuda.synchronize()
    return out, kc, vc


def check(c, got, slots=None):
    out, kc, vc = (x.double().cpu().numpy() for x in got)
    t, dim = c["q"].shape[0], c["dim"]
    pos = c["positions"].cpu().numpy()
    slots = c["slots"].cpu().numpy() if slots is None else slots
    keep = slots >= 0

    def plain(x, w, rotate=True):
        x = x.float().cpu().numpy().reshape(t, -1, dim)
        return attn_plain.norm_rope(x, None if w is None else w.cpu().numpy(), c["cos"].cpu().numpy(),
                                    c["sin"].cpu().numpy(), pos, c["rot"], c["half"], c["eps"], rotate)

    for name, have, (want, size) in (("q", out, plain(c["q"], c["wq"])),
                                     ("k", kc[slots[keep]], [y[keep] for y in plain(c["k"], c["wk"])]),
                                     ("v", vc[slots[keep]], [y[keep] for y in plain(c["v"], None, False)])):
        bound = attn_plain.norm_rope_bound(want, size, c["dtype"], dim)
        assert np.all(np.abs(have - want) <= bound), name
    # the other slots are as they were
    rest = np.setdiff1d(np.arange(kc.shape[0]), slots)
    assert np.array_equal(kc[rest], c["kc"].double().cpu().numpy()[rest])
    assert np.array_equal(vc[rest], c["vc"].double().cpu().numpy()[rest])


@pytest.mark.parametrize("t,hq,hkv,dim,kw", [
    (1, 1, 1, 64, {}), (1, 32, 8, 128, {}), (3, 64, 8, 128, dict(dtype=FP)), (17, 5, 1, 64, dict(norm=(False, False))),
    (40, 8, 2, 128, dict(half=False)), (40, 6, 3, 64, dict(half=False, norm=(True, False))),
    (33, 7, 1, 128, dict(rot=64)), (9, 4, 4, 64, dict(rot=24, half=False)), (9, 4, 4, 128, dict(rot=40)),
    (5, 3, 1, 128, dict(rot=0)), (5, 3, 1, 64, dict(rot=8, norm=(False, True))),
    (21, 8, 2, 128, dict(fused=True)), (21, 9, 3, 64, dict(fused=True, dtype=FP)),
    (13, 8, 2, 128, dict(in_dtype=BF)), (13, 8, 2, 64, dict(in_dtype=FP, dtype=FP)),
    (13, 8, 2, 128, dict(in_dtype=FP, dtype=BF)), (13, 8, 2, 128, dict(in_dtype=BF, dtype=FP, fused=True)),
    (2000, 12, 2, 128, {}), (3001, 2, 1, 64, dict(norm=(False, False))),
])
def test_against_64_bits(t, hq, hkv, dim, kw):
    c = make(t, hq, hkv, dim, seed=t + hq, **kw)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    check(c, call(c, status))
    assert int(status) == 0


def test_tokens_that_are_not_kept_and_packed_keys():
    c = make(30, 4, 2, 128, seed=5)
    c["slots"][::3] = -1
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    check(c, call(c, status))
    assert int(status) == 0
    check(c, call(c, slots=None), slots=np.arange(30))


def test_zero_and_extreme_rows():
    c = make(6, 2, 1, 64, seed=6)
    c["q"][0] = 0.0
    c["q"][1] = 1e15
    c["q"][2] = 1e-18
    out, _, _ = call(c)
    assert torch.all(out[0] == 0)
    check(c, call(c))


def test_a_nan_stays_in_its_head():
    c = make(4, 4, 2, 128, seed=7)
    clean = call(c)
    c["q"][1, 128 + 5] = float("nan")
    got = call(c)
    assert torch.isnan(got[0][1, 1]).any()
    same = torch.ones((4, 4), dtype=torch.bool)
    same[1, 1] = False
    assert torch.equal(got[0][same.to(DEV)], clean[0][same.to(DEV)])
    assert torch.equal(got[1], clean[1]) and torch.equal(got[2], clean[2])


def test_positions_and_slots_out_of_range():
    c = make(8, 4, 2, 64, seed=8)
    good = call(c)
    for bad in (c["kc"].shape[0], 2 ** 31 - 1):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        d = dict(c, slots=c["slots"].clone())
        d["slots"][3] = bad
        out, kc, vc = call(d, status)
        assert int(status) == sss.FLAG_INDEX
        assert torch.equal(out, good[0])
        row = int(c["slots"][3])
        assert torch.equal(kc[row], c["kc"][row]) and torch.equal(vc[row], c["vc"][row])
    for bad, taken in ((-1, 0), (500, 499), (2 ** 31 - 1, 499)):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        d = dict(c, positions=c["positions"].clone())
        d["positions"][2] = bad
        got = call(d, status)
        assert int(status) == sss.FLAG_INDEX
        d["positions"][2] = taken
        for g, w in zip(got, call(d)):
            assert torch.equal(g, w)


def test_other_stream_and_offsets_past_32_bits():
    c = make(50, 8, 2, 128, seed=9)
    want = call(c)
    for g, w in zip(call(c, stream=torch.cuda.Stream()), want):
        assert torch.equal(g, w)
    slots = 2 ** 31 // 256 + 100
    kc, vc = (torch.zeros((slots, 2, 128), dtype=BF, device=DEV) for _ in range(2))
    far = c["slots"] + (slots - 1 - int(c["slots"].max()))
    sss.sss_qk_norm_rope(c["q"], c["k"], c["v"], sss.Rope(c["cos"], c["sin"], 0, c["wq"], c["wk"], c["eps"]),
                         c["positions"], sss.KVCache(kc, vc, 16), slots=far)
    torch.cuda.synchronize()
    at = c["slots"].long()
    assert torch.equal(kc[far.long()], want[1][at]) and torch.equal(vc[far.long()], want[2][at])


def test_empty_and_python_refusals():
    c = make(4, 4, 2, 64, seed=10)
    cache = sss.KVCache(c["kc"], c["vc"], 16)
    rope = sss.Rope(c["cos"], c["sin"], 0, c["wq"], c["wk"])
    a = dict(q=c["q"], k=c["k"], v=c["v"], rope=rope, positions=c["positions"], cache=cache, slots=c["slots"])
    assert sss.sss_qk_norm_rope(**{**a, **{n: a[n][:0] for n in ("q", "k", "v", "positions", "slots")}}).numel() == 0
    bad = [
        (dict(q=c["q"].half()), "dtype"), (dict(q=c["q"][:, :100]), "heads"), (dict(k=c["k"][:2]), "k must be"),
        (dict(v=c["v"].t().contiguous().t()), "contiguous"), (dict(positions=c["positions"].long()), "int32"),
        (dict(positions=None), "required"), (dict(slots=c["slots"][:2]), "elements"), (dict(k=c["k"].cpu()), "CUDA"),
        (dict(q_out=torch.empty((4, 4, 64), dtype=F32, device=DEV)), "bfloat16"),
        (dict(rope=sss.Rope(c["cos"], c["sin"], 2)), "SSS_E_ARG"),
        (dict(rope=sss.Rope(c["cos"], c["sin"], 0, eps=-1.0)), "SSS_E_ARG"),
        (dict(rope=sss.Rope(c["cos"][:, :3].contiguous(), c["sin"][:, :3].contiguous())), "SSS_E_ARG"),
        (dict(rope=sss.Rope(c["cos"], c["sin"], 0, torch.ones(32, device=DEV))), "elements"),
    ]
    for change, what in bad:
        with pytest.raises(sss.SssError, match=what):
            sss.sss_qk_norm_rope(**{**a, **change})
