"""Host-side argument checks of sss_page_plan, sss_qk_norm_rope and sss_attention:
the documented status codes, before any CUDA call (no GPU here)."""
import ctypes

import pytest

from paper_2607_08779_gb300 import sss

P = 4096  # a 16-byte aligned address that nothing reads


def cache(**kw):
    a = dict(k=P, v=P, slots=64, stride=256, page_size=16, heads=2, dim=128, dtype=sss.OUT_BF16)
    a.update(kw)
    return sss.KVCacheDesc(*[a[n] for n, _ in sss.KVCacheDesc._fields_])


def attention(c=None, **kw):
    a = dict(q=P, q_stride=512, heads=4, cu=P, kv=P, table=P, width=4, batch=0, tokens=0, max_q=1, max_kv=64,
             scale=0.1, out=P, ws=None, ws_bytes=0, status=None)
    a.update(kw)
    return sss.load().sss_attention(a["q"], a["q_stride"], a["heads"], ctypes.byref(c or cache()), a["cu"], a["kv"],
                                    a["table"], a["width"], a["batch"], a["tokens"], a["max_q"], a["max_kv"],
                                    a["scale"], a["out"], a["ws"], a["ws_bytes"], a["status"], None)


full = dict(batch=1, tokens=1)
many = dict(batch=1, tokens=64, max_q=64)


@pytest.mark.parametrize("kw,want", [
    (dict(), 0),                                        # an empty call touches nothing
    (dict(tokens=5, batch=0), 0), (dict(full, max_q=0), 0),
    (dict(heads=3), 1), (dict(heads=0), 1), (dict(q_stride=504), 1), (dict(q_stride=516), 1),
    (dict(batch=-1), 1), (dict(tokens=-1), 1), (dict(tokens=1 << 25), 1), (dict(max_q=-1), 1), (dict(max_kv=-1), 1),
    (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=float("inf")), 1), (dict(scale=float("nan")), 1),
    (dict(width=0), 1), (dict(kv=None), 1),
    (dict(full, q=None), 1), (dict(full, out=None), 1), (dict(full, cu=None), 1),
    (dict(full, q=P + 8), 3), (dict(full, out=P + 2), 3), (dict(full, cu=P + 2), 3), (dict(full, table=P + 1), 3),
    (dict(many, max_kv=100000), 5), (dict(many, max_kv=100000, ws=P, ws_bytes=100), 5),
    (dict(many, max_kv=100000, ws=P + 8, ws_bytes=1 << 30), 3),
])
def test_attention_arguments(kw, want):
    assert attention(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(dim=96), 2), (dict(dim=256, stride=512), 2), (dict(dim=0), 1), (dict(dtype=sss.OUT_F32), 1), (dict(dtype=3), 1),
    (dict(heads=0), 1), (dict(slots=-1), 1), (dict(slots=1 << 31), 1), (dict(stride=248), 1), (dict(stride=260), 1),
    (dict(k=None), 1), (dict(k=P + 8), 3), (dict(v=P + 2), 3), (dict(page_size=8), 1), (dict(page_size=48), 1),
    (dict(page_size=512), 1),
])
def test_cache_descriptors(kw, want):
    assert attention(cache(**kw)) == want


def test_page_size_does_not_matter_without_a_table():
    assert attention(cache(page_size=7), table=None, kv=None) == 0


def test_attention_workspace():
    L = sss.load()
    c = cache(heads=8, stride=1024)
    size = lambda *a: L.sss_attention_workspace_bytes(a[0], a[1], ctypes.byref(c), *a[2:])  # noqa: E731
    assert size(1, 32, 1, 1, 16) == 0            # nothing to split
    assert size(64, 32, 1, 64, 8192) > 64 * 32 * 128 * 4  # partial rows
    assert size(0, 32, 1, 64, 8192) == 0 and size(64, 32, 0, 64, 8192) == 0
    assert size(64, 31, 1, 64, 8192) == 0 and size(-1, 32, 1, 64, 8192) == 0 and size(64, 32, 1, 64, -1) == 0


def test_page_plan_arguments():
    def plan(**kw):
        a = dict(past=P, fresh=P, batch=2, page=16, free=P, nfree=3, table=P, width=4, cu=P, kv=P, pos=P, slots=P,
                 tokens=2, used=P, status=None)
        a.update(kw)
        return sss.load().sss_page_plan(a["past"], a["fresh"], a["batch"], a["page"], a["free"], a["nfree"], a["table"],
                                        a["width"], a["cu"], a["kv"], a["pos"], a["slots"], a["tokens"], a["used"],
                                        a["status"], None)

    for kw in (dict(batch=-1), dict(page=0), dict(page=24), dict(page=512), dict(nfree=-1), dict(width=-1),
               dict(tokens=-1), dict(past=None), dict(fresh=None), dict(table=None), dict(free=None), dict(cu=None),
               dict(kv=None), dict(pos=None), dict(slots=None), dict(used=None)):
        assert plan(**kw) == 1, kw
    for name in ("past", "fresh", "free", "table", "cu", "kv", "pos", "slots", "used", "status"):
        assert plan(**{name: P + 2}) == 3, name


def test_qk_norm_rope_arguments():
    def rope(c=None, r=None, **kw):
        d = dict(cos=P, sin=P, q_norm=None, k_norm=None, max_pos=10, rot_dim=128, style=0, eps=1e-6)
        d.update(r or {})
        desc = sss.RopeDesc(*[d[n] for n, _ in sss.RopeDesc._fields_])
        a = dict(q=P, qs=512, k=P, ks=256, v=P, vs=256, dt=0, tokens=3, heads=4, pos=P, out=P, slots=P, status=None)
        a.update(kw)
        return sss.load().sss_qk_norm_rope(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["dt"], a["tokens"],
                                           a["heads"], ctypes.byref(desc), a["pos"], a["out"],
                                           ctypes.byref(c or cache()), a["slots"], a["status"], None)

    assert rope(tokens=0) == 0
    assert rope(tokens=0, q=None, pos=None) == 0
    for kw in (dict(qs=508), dict(ks=252), dict(vs=255), dict(qs=514), dict(dt=3), dict(dt=-1), dict(tokens=-1),
               dict(heads=0), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(pos=None)):
        assert rope(**kw) == 1, kw
    for r in (dict(rot_dim=136), dict(rot_dim=-8), dict(rot_dim=20), dict(style=2), dict(eps=-1.0), dict(eps=float("nan")),
              dict(max_pos=0), dict(max_pos=-1), dict(cos=None), dict(sin=None)):
        assert rope(r=r) == 1, r
    for kw in (dict(q=P + 8), dict(k=P + 4), dict(out=P + 8), dict(pos=P + 2), dict(slots=P + 1), dict(status=P + 1)):
        assert rope(**kw) == 3, kw
    assert rope(q=P + 8, k=P + 8, v=P + 8, dt=sss.OUT_BF16, slots=P + 2) == 3
    for r in (dict(cos=P + 4), dict(sin=P + 8), dict(q_norm=P + 4), dict(k_norm=P + 8)):
        assert rope(r=r) == 3, r
    assert rope(cache(dim=256, stride=512)) == 2


def test_python_cache_and_rope_refusals():
    torch = pytest.importorskip("torch")
    k = torch.zeros((32, 2, 64), dtype=torch.bfloat16)
    for a, b, what in ((k, k[:16], "shape"), (k[0], k[0], "slots"), (k.float(), k.float(), "float16"),
                       (k, k.half(), "float16"), (k[..., ::2], k[..., ::2], "contiguous"), (k, k, "CUDA"),
                       (torch.zeros((32, 4, 64), dtype=torch.bfloat16)[:, :2], k, "stride")):
        with pytest.raises(sss.SssError, match=what):
            sss.KVCache(a, b)
    cos = torch.zeros((8, 32))
    for kw, what in ((dict(cos=cos), "together"), (dict(cos=cos, sin=cos[:4]), "max_pos"),
                     (dict(cos=cos.double(), sin=cos.double()), "float32"), (dict(cos=cos, sin=cos), "CUDA")):
        with pytest.raises(sss.SssError, match=what):
            sss.Rope(**kw)


@pytest.mark.parametrize("kw,want", [
    (dict(heads=16384, q_stride=16384 * 128), 0), (dict(heads=16386, q_stride=16386 * 128), 1),
    (dict(batch=65536), 1), (dict(max_kv=1 << 31), 1),
])
def test_the_largest_attention(kw, want):
    assert attention(**kw) == want
