"""A serving loop of beams over both caches with all of the pages' operators in it: rows
forked from their parents, their last pages copied, free pages found again, held ones
moved down, pages planned, keys and values stored, attention; eagerly and as one captured
graph that is replayed, without anything read back.  Each step's rows are compared with plain
attention over what each beam has seen."""
import numpy as np
import pytest
import torch

import attn_plain
import q4_plain
from paper_2607_08779_gb300 import sss

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device=DEV)


class Loop:
    """The buffers and one step of `rows` beams with one new token each."""

    def __init__(self, rows, hq, hkv, dim, page, pages, width, layers, most):
        self.page, self.most, self.max_kv = page, most, width * page
        self.table, self.new_table = ints(rows, width).fill_(-1), ints(rows, width)
        self.past, self.new_past, self.kv_len, self.parents = ints(rows), ints(rows), ints(rows), ints(rows)
        self.fresh = ints(rows).fill_(1)
        self.src, self.dst, self.used, self.status = ints(rows), ints(rows), ints(1), ints(1)
        self.free, self.count = torch.arange(pages, dtype=torch.int32, device=DEV), ints(1)
        self.msrc, self.mdst, self.moves = ints(most), ints(most), ints(1)
        self.cu_q, self.positions, self.slots = ints(rows + 1), ints(rows), ints(rows)
        self.q4 = [sss.empty_kv_cache_q4(pages, page, hkv, dim) for _ in range(layers)]
        self.c16 = [sss.empty_kv_cache(pages, page, hkv, dim) for _ in range(layers)]
        self.q = torch.zeros((layers, rows, hq, dim), dtype=BF, device=DEV)
        self.k, self.v = (torch.zeros((layers, rows, hkv, dim), dtype=BF, device=DEV) for _ in range(2))
        self.out4, self.out16 = torch.zeros_like(self.q), torch.zeros_like(self.q)
        self.rope = sss.Rope()  # (no rotation: what is stored is what came)
        self.turned = torch.zeros_like(self.q)

    def step(self):
        st = self.status
        sss.sss_page_fork(self.parents, self.past, self.page, self.free, self.table, self.new_table, self.new_past, self.src,
                          self.dst, self.used, dev_status=st)
        sss.sss_page_copy(self.q4, self.src, self.dst, dev_status=st)
        sss.sss_page_copy(self.c16, self.src, self.dst, dev_status=st)
        sss.sss_page_reclaim(self.new_table, self.new_past, self.page, self.free, self.count, self.new_table, self.msrc,
                             self.mdst, self.moves, dev_status=st)
        sss.sss_page_copy(self.q4, self.msrc, self.mdst, dev_status=st)
        sss.sss_page_copy(self.c16, self.msrc, self.mdst, dev_status=st)
        sss.sss_page_plan(self.new_past, self.fresh, self.page, self.free, self.new_table, self.cu_q, self.kv_len,
                          self.positions, self.slots, self.used, dev_status=st)
        for i, (c4, c16) in enumerate(zip(self.q4, self.c16)):
            rows = self.q.shape[1]
            sss.sss_qk_norm_rope(self.q[i].view(rows, -1), self.k[i].view(rows, -1), self.v[i].view(rows, -1), self.rope, None,
                                 c16, slots=self.slots, q_out=self.turned[i], dev_status=st)
            sss.sss_kv_store_q4(self.k[i], self.v[i], c4, self.slots, dev_status=st)
            args = (self.cu_q, self.kv_len, 1, self.max_kv)
            sss.sss_attention(self.turned[i], c16, *args, block_table=self.new_table, out=self.out16[i], dev_status=st)
            sss.sss_attention_q4(self.turned[i], c4, *args, self.new_table, out=self.out4[i], dev_status=st)
        # the free pages, now that the step's are taken
        sss.sss_page_reclaim(self.new_table, self.kv_len, self.page, self.free, self.count, dev_status=st)
        self.table.copy_(self.new_table)
        self.past.copy_(self.kv_len)


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("rows,hq,hkv,dim,page,steps,most", [(6, 8, 2, 128, 16, 40, 100), (4, 4, 4, 64, 32, 70, 1),
                                                            (9, 16, 1, 128, 16, 36, 0)])
def test_beams_see_their_own_past(captured, rows, hq, hkv, dim, page, steps, most):
    layers, width = 2, -(-steps // page) + 1
    pages = rows * (width + 2)
    rng = np.random.default_rng(rows)
    g = torch.Generator().manual_seed(rows)
    loop = Loop(rows, hq, hkv, dim, page, pages, width, layers, most)
    graph = None
    if captured:
        loop.step()  # (the kernels' first calls)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            loop.step()
        loop.table.fill_(-1)
        loop.past.zero_()
        loop.free.copy_(torch.arange(pages, dtype=torch.int32))
        loop.status.zero_()
    past = [[] for _ in range(rows)]  # per beam: the numbers of the tokens that it has seen
    seen = [[], [], []]               # all tokens' keys and values
    for step in range(steps):
        parents = rng.integers(0, rows, rows) if step % 3 else np.arange(rows)
        if step % 7 == 5:
            parents[0] = -1           # a beam that starts anew
        q = torch.randn((layers, rows, hq, dim), generator=g).to(BF)
        k, v = (torch.randn((layers, rows, hkv, dim), generator=g).to(BF) for _ in range(2))
        loop.parents.copy_(torch.from_numpy(parents.astype(np.int32)))
        loop.q.copy_(q)
        loop.k.copy_(k)
        loop.v.copy_(v)
        if graph is None:
            loop.step()
        else:
            graph.replay()
        past = [(past[p] if p >= 0 else []) + [step * rows + r] for r, p in enumerate(parents)]
        seen[0].append(k)
        seen[1].append(v)
        if step % 5 and step != steps - 1:
            continue
        torch.cuda.synchronize()
        assert int(loop.status) == 0
        assert loop.past.tolist() == [len(p) for p in past]
        # every page of the tables is held by rows that share it, and no other is missing
        held = {int(x) for r in range(rows) for x in loop.table[r, :-(-len(past[r]) // page)]}
        assert sorted(held | set(loop.free[:int(loop.count)].tolist())) == list(range(pages))
        assert not held & set(loop.free[:int(loop.count)].tolist())
        if most == 100:  # (before the step's new pages they are the lowest)
            assert max(held) < len(held) + rows
        keys, values = (torch.cat(x, dim=1) for x in seen[:2])  # [layers, tokens, hkv, dim]
        kv, cu = [len(p) for p in past], list(range(rows + 1))
        for i in range(layers):
            rows_of = lambda b: np.array(past[b])  # noqa: E731
            w = attn_plain.attention(q[i], keys[i], values[i], cu, kv, rows_of, dim ** -0.5)
            err = np.abs(loop.out16[i].cpu().double().numpy() - w[0])
            assert np.max(err / attn_plain.attention_bound(*w, BF, max(kv))) <= 1.0
            packed = [q4_plain.quantize(x[i].float().numpy()) for x in (keys, values)]
            w = q4_plain.attention(q[i], *[(q4_plain.values(u, s), s) for u, s, _ in packed], cu, kv, rows_of, dim ** -0.5)
            err = np.abs(loop.out4[i].cpu().double().numpy() - w["out"])
            assert np.max(err / q4_plain.bound_rows(w, BF, dim, max(kv))) <= 1.0


def test_prompts_then_tokens_and_back():
    """A prompt attends to its packed 16-bit keys, then goes into the 4-bit cache; a chunk
    and single tokens go on from there.  A request then ends and its pages are free."""
    hq, hkv, dim, page, lens = 8, 2, 128, 16, [70, 33]
    g = torch.Generator(device=DEV).manual_seed(3)
    cache, status = sss.empty_kv_cache_q4(20, page, hkv, dim), ints(1)
    table, free, count = ints(2, 12).fill_(-1), torch.arange(20, dtype=torch.int32, device=DEV), ints(1)
    past, keys, values = ints(2), [[], []], [[], []]
    for fresh in (lens, [20, 1], [1, 1]):
        t = sum(fresh)
        q = torch.randn((t, hq, dim), generator=g, device=DEV).to(BF)
        k, v = (torch.randn((t, hkv, dim), generator=g, device=DEV).to(BF) for _ in range(2))
        cu, kv, positions, slots, used = ints(3), ints(2), ints(t), ints(t), ints(1)
        sss.sss_page_plan(past, torch.tensor(fresh, dtype=torch.int32, device=DEV), page, free, table, cu, kv, positions, slots,
                          used, dev_status=status)
        sss.sss_kv_store_q4(k, v, cache, slots, dev_status=status)
        out = sss.sss_attention_q4(q, cache, cu, kv, max(fresh), 200, table, dev_status=status)
        for b, (x, y) in enumerate(zip(k.split(fresh), v.split(fresh))):
            keys[b].append(x.cpu())
            values[b].append(y.cpu())
        kvs = kv.tolist()
        packed = [q4_plain.quantize(torch.cat([torch.cat(x) for x in z]).float().numpy()) for z in (keys, values)]
        at = [0, kvs[0]]
        w = q4_plain.attention(q.cpu(), *[(q4_plain.values(u, s), s) for u, s, _ in packed], cu.tolist(), kvs,
                               lambda b: at[b] + np.arange(kvs[b]), dim ** -0.5)
        bound = q4_plain.bound_many if max(fresh) * hq // hkv > 64 else q4_plain.bound_rows
        err = np.abs(out.cpu().double().numpy() - w["out"])
        assert np.max(err / bound(w, BF, dim, 200)) <= 1.0
        past.copy_(kv)
        sss.sss_page_reclaim(table, past, page, free, count, dev_status=status)
        assert int(count) == 20 - sum(-(-n // page) for n in kvs)
    past[0] = 0  # it has ended
    sss.sss_page_reclaim(table, past, page, free, count, dev_status=status)
    assert int(count) == 20 - -(-int(past[1]) // page) and int(status) == 0


def test_the_same_bits_without_the_compiled_binding(monkeypatch):
    def run():
        loop = Loop(4, 8, 2, 128, 16, 40, 4, 2, 8)
        g = torch.Generator(device=DEV).manual_seed(9)
        for step in range(20):
            loop.parents.copy_(torch.tensor([(step * r) % 4 for r in range(4)], dtype=torch.int32))
            for x in (loop.q, loop.k, loop.v):
                x.copy_(torch.randn(x.shape, generator=g, device=DEV))
            loop.step()
        a = loop.k[0].clone(), loop.v[0].clone()
        fetched = sss.sss_kv_fetch_q4(loop.q4[0], loop.slots, *a)
        torch.cuda.synchronize()
        assert int(loop.status) == 0
        return [loop.out4, loop.out16, loop.table, loop.free, loop.count, *fetched]

    assert sss._binding() is not sss._NoBinding  # (it is there on this machine)
    with_it = run()
    monkeypatch.setattr(sss, "_fast", sss._NoBinding)
    for x, y in zip(with_it, run()):
        assert torch.equal(x, y)
