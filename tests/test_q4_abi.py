"""Host-side argument checks of the 4-bit cache's and the shared pages' calls, before any
CUDA call, and of the plain forms that their results are compared with (no GPU here)."""
import ctypes

import numpy as np
import pytest

import q4_plain
from paper_2607_08779_gb300 import sss

P = 4096  # a 16-byte aligned address that nothing reads


def cache(**kw):
    a = dict(blocks=P, pages=4, page_stride=2 * 18 * 128, page_size=16, heads=2, dim=128, reserved=0)
    a.update(kw)
    return sss.KVCacheQ4Desc(*[a[n] for n, _ in sss.KVCacheQ4Desc._fields_])


def store(c=None, **kw):
    a = dict(k=P, ks=256, v=P, vs=256, dt=sss.OUT_BF16, tokens=1, slots=P, status=None)
    a.update(kw)
    return sss.load().sss_kv_store_q4(a["k"], a["ks"], a["v"], a["vs"], a["dt"], a["tokens"], ctypes.byref(c or cache()),
                                      a["slots"], a["status"], None)


def fetch(c=None, **kw):
    a = dict(slots=P, count=1, k=P, v=P, dt=sss.OUT_BF16, status=None)
    a.update(kw)
    return sss.load().sss_kv_fetch_q4(ctypes.byref(c or cache()), a["slots"], a["count"], a["k"], a["v"], a["dt"],
                                      a["status"], None)


def attention(c=None, **kw):
    a = dict(q=P, q_stride=512, heads=4, dt=sss.OUT_BF16, cu=P, kv=P, table=P, width=4, batch=0, tokens=0, max_q=1,
             max_kv=64, scale=0.1, out=P, ws=None, ws_bytes=0, status=None)
    a.update(kw)
    return sss.load().sss_attention_q4(a["q"], a["q_stride"], a["heads"], a["dt"], ctypes.byref(c or cache()), a["cu"],
                                       a["kv"], a["table"], a["width"], a["batch"], a["tokens"], a["max_q"], a["max_kv"],
                                       a["scale"], a["out"], a["ws"], a["ws_bytes"], a["status"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(), 0), (dict(dim=64), 0), (dict(dim=96), 2), (dict(dim=256, page_stride=1 << 20), 2), (dict(dim=0), 1),
    (dict(heads=0), 1), (dict(heads=3), 1), (dict(pages=-1), 1), (dict(pages=1 << 27), 1), (dict(page_size=8), 1),
    (dict(page_size=32), 1), (dict(page_size=48, page_stride=1 << 20), 1), (dict(page_stride=2 * 18 * 128 + 8), 1),
    (dict(page_stride=2 * 18 * 128 - 16), 1), (dict(page_stride=1 << 41), 1), (dict(blocks=None), 1),
    (dict(blocks=None, pages=0), 0), (dict(blocks=P + 8), 3), (dict(reserved=1), 1),
])
def test_cache_descriptors(kw, want):
    assert store(cache(**kw), tokens=0) == want
    assert fetch(cache(**kw), count=0) == want
    assert attention(cache(**kw), heads=6 if kw.get("heads") == 3 else 4, q_stride=1024) == want


def test_store_and_fetch_arguments():
    for kw in (dict(ks=248), dict(vs=255), dict(ks=260), dict(dt=3), dict(dt=-1), dict(tokens=-1), dict(tokens=1 << 25),
               dict(k=None), dict(v=None)):
        assert store(**kw) == 1, kw
    for kw in (dict(k=P + 8), dict(v=P + 4), dict(slots=P + 2), dict(status=P + 1)):
        assert store(**kw) == 3, kw
    assert store(tokens=0, k=None, v=None, slots=None) == 0
    for kw in (dict(dt=3), dict(count=-1), dict(count=1 << 25)):
        assert fetch(**kw) == 1, kw
    for kw in (dict(k=P + 8), dict(v=P + 2), dict(slots=P + 2), dict(status=P + 1)):
        assert fetch(**kw) == 3, kw
    assert fetch(count=0, slots=None) == 0 and fetch(k=None, v=None) == 0


full = dict(batch=1, tokens=1)
many = dict(batch=1, tokens=64, max_q=64)


@pytest.mark.parametrize("kw,want", [
    (dict(), 0), (dict(tokens=5, batch=0), 0), (dict(full, max_q=0), 0),
    (dict(heads=3), 1), (dict(heads=0), 1), (dict(q_stride=504), 1), (dict(q_stride=516), 1), (dict(dt=0), 1), (dict(dt=3), 1),
    (dict(batch=-1), 1), (dict(batch=65536), 1), (dict(tokens=-1), 1), (dict(tokens=1 << 25), 1), (dict(max_q=-1), 1),
    (dict(max_kv=-1), 1), (dict(max_kv=1 << 31), 1), (dict(width=0), 1),
    (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=2.4e38), 1), (dict(scale=float("nan")), 1),
    (dict(full, q=None), 1), (dict(full, out=None), 1), (dict(full, cu=None), 1), (dict(full, kv=None), 1),
    (dict(full, table=None), 1), (dict(full, q=P + 8), 3), (dict(full, out=P + 2), 3), (dict(full, cu=P + 2), 3),
    (dict(full, table=P + 1), 3), (dict(full, kv=P + 2), 3), (dict(full, status=P + 2), 3),
    (dict(many), 5), (dict(many, ws=P, ws_bytes=100), 5), (dict(many, ws=P + 8, ws_bytes=1 << 30), 3),
    (dict(batch=65535, tokens=65535, max_q=64, max_kv=1 << 20, width=1 << 16), 2),  # the copy would have 2^36 slots
])
def test_attention_arguments(kw, want):
    assert attention(**kw) == want


def test_attention_workspace():
    c = cache(heads=8, page_stride=8 * 18 * 128)
    size = lambda t, h, w, b, mq, mkv: sss.load().sss_attention_q4_workspace_bytes(t, h, ctypes.byref(c), w, b, mq, mkv)  # noqa: E731
    assert size(64, 32, 100, 64, 1, 1600) == 0               # single tokens read the cache as it is
    assert size(64, 32, 999, 64, 1, 16000) == 8 * 64 * 32 * (128 + 1) * 4  # long ones leave a chunk's results each
    copy = 2 * 1600 * 8 * 128 * 2
    assert copy <= size(64, 32, 100, 1, 64, 1600) < 2 * copy + (1 << 20) * 64
    assert size(64, 32, 50, 1, 64, 1600) < size(64, 32, 100, 1, 64, 1600) == size(64, 32, 2 ** 31 - 1, 1, 64, 1600)
    assert size(64, 32, 100, 1, 10 ** 9, 1600) == size(64, 32, 100, 1, 64, 1600)
    assert size(64, 31, 100, 1, 64, 1600) == size(-1, 32, 100, 1, 64, 1600) == size(64, 32, 0, 1, 64, 1600) == 0


def test_fork_arguments():
    def fork(**kw):
        a = dict(parents=P, rows=2, past=P, batch=2, page=16, free=P, nfree=1, table=P, width=2, new=2 * P, new_past=2 * P,
                 src=P, dst=P, used=P, status=None)
        a.update(kw)
        return sss.load().sss_page_fork(*[a[n] for n in ("parents", "rows", "past", "batch", "page", "free", "nfree", "table",
                                                         "width", "new", "new_past", "src", "dst", "used", "status")], None)

    for kw in (dict(rows=-1), dict(rows=65536), dict(batch=-1), dict(batch=65536), dict(page=24), dict(page=0), dict(nfree=-1),
               dict(width=-1), dict(parents=None), dict(past=None), dict(free=None), dict(table=None), dict(new=None),
               dict(new_past=None), dict(src=None), dict(dst=None), dict(used=None), dict(new=P), dict(new_past=P)):
        assert fork(**kw) == 1, kw
    for name in ("parents", "past", "free", "table", "new", "new_past", "src", "dst", "used", "status"):
        assert fork(**{name: 4 * P + 2}) == 3, name


def test_reclaim_arguments():
    def reclaim(**kw):
        a = dict(table=P, width=2, past=P, batch=2, page=16, pages=10, free=P, count=P, new=P, src=P, dst=P, most=3, moves=P,
                 status=None)
        a.update(kw)
        return sss.load().sss_page_reclaim(*[a[n] for n in ("table", "width", "past", "batch", "page", "pages", "free", "count",
                                                            "new", "src", "dst", "most", "moves", "status")], None)

    for kw in (dict(width=-1), dict(batch=-1), dict(page=17), dict(pages=-1), dict(pages=(1 << 20) + 1), dict(most=-1),
               dict(table=None), dict(past=None), dict(free=None), dict(count=None), dict(src=None), dict(dst=None),
               dict(moves=None), dict(new=None)):
        assert reclaim(**kw) == 1, kw
    for name in ("table", "past", "free", "count", "new", "src", "dst", "moves", "status"):
        assert reclaim(**{name: P + 2}) == 3, name


def test_copy_arguments():
    L = sss.load()
    c16 = lambda **kw: sss.KVCacheDesc(*[{**dict(k=P, v=P, slots=64, stride=256, page_size=16, heads=2, dim=128,  # noqa: E731
                                                 dtype=sss.OUT_BF16), **kw}[n] for n, _ in sss.KVCacheDesc._fields_])

    def copy(f, caches, count=None, src=P, dst=P, n=0, status=None):
        at = (ctypes.c_void_p * max(1, len(caches)))(*[ctypes.addressof(c) for c in caches])
        return f(at, len(caches) if count is None else count, src, dst, n, status, None)

    for f, good, others in ((L.sss_page_copy, c16, (dict(page_size=32), dict(heads=1), dict(dim=64), dict(slots=80))),
                            (L.sss_page_copy_q4, cache, (dict(page_size=32, page_stride=1 << 20), dict(heads=1), dict(dim=64),
                                                         dict(pages=5)))):
        assert copy(f, [good()]) == 0 and copy(f, []) == 0 and copy(f, [], src=None, dst=None) == 0
        assert copy(f, [good()], n=-1) == 1 and copy(f, [good()], count=-1) == 1 and copy(f, [good()] * 129) == 1
        assert copy(f, [good()], src=None, n=1) == 1 and copy(f, [good()], dst=None, n=1) == 1
        assert copy(f, [good()], src=P + 2, n=1) == 3 and copy(f, [good()], status=P + 2) == 3
        for kw in others:
            assert copy(f, [good(), good(**kw)]) == 1, kw
        assert f(None, 1, P, P, 1, None, None) == 1
    assert copy(L.sss_page_copy, [c16(page_size=7)]) == 1
    assert copy(L.sss_page_copy, [c16(k=P + 8)]) == 3 and copy(L.sss_page_copy_q4, [cache(blocks=P + 8)]) == 3


def test_python_cache_refusals():
    torch = pytest.importorskip("torch")
    t = torch.zeros((4, 2, 1, 18 * 64), dtype=torch.uint8)
    for bad, what in ((t[0], "uint8"), (t.float(), "uint8"), (t[..., :100], "18"), (t[:, :, :, ::2], "18|contiguous"),
                      (t, "CUDA"), (torch.zeros((4, 4, 1, 18 * 64), dtype=torch.uint8)[:, ::2], "contiguous")):
        with pytest.raises(sss.SssError, match=what):
            sss.KVCacheQ4(bad)
    with pytest.raises(sss.SssError, match="multiple"):
        sss.empty_kv_cache_q4(4, 24, 2, 64, device="cpu")


@pytest.mark.parametrize("dim", [64, 128])
def test_a_word_holds_each_dimension_once(dim):
    # the layout is a permutation: a code of 1 in one place sets one nibble, each another
    seen = set()
    for d in range(dim):
        u = np.zeros((1, 1, dim), np.uint8)
        u[0, 0, d] = 1
        words = q4_plain.pack(u, dim)[0, 0]
        (w,) = np.nonzero(words)[0]
        seen.add((int(w), int(words[w])))
    assert len(seen) == dim and all(bin(v).count("1") == 1 and v & 0x11111111 for _, v in seen)


def test_plain_fork_and_reclaim():
    table = np.array([[5, 6, -1], [7, -1, -1]])
    new, past, src, dst, used = q4_plain.fork([0, 0, 1, -1, 1], [20, 16], 16, [9, 8], table)
    assert new.tolist() == [[5, 6, -1], [5, 9, -1], [7, -1, -1], [-1] * 3, [7, -1, -1]]
    assert past.tolist() == [20, 20, 16, 0, 16] and src.tolist() == [-1, 6, -1, -1, -1]
    assert dst.tolist() == [-1, 9, -1, -1, -1] and used.tolist() == [1]
    free, count, new, src, dst, moves = q4_plain.reclaim(table, [20, 16], 16, 9, 8)
    assert src.tolist()[:3] == [7, 6, 5] and dst.tolist()[:3] == [0, 1, 2] and moves.tolist() == [3]
    assert free.tolist() == [3, 4, 5, 6, 7, 8, -1, -1, -1] and new.tolist() == [[2, 1, -1], [0, -1, -1]]
