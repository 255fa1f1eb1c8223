"""Drafted tokens over the 4-bit cache: each step forks the rows of the block table, copies their
last pages, plans the new tokens' pages, normalises and rotates them into a 16-bit buffer, stores that
in 4 bits and attends; then rows are cut back, by rejected tokens or to anywhere, also into pages
that others share.  Eagerly and as one captured graph; what each row attends to is its own."""
import numpy as np
import pytest
import torch

import attn_plain
import q4_plain
from paper_2607_08779_gb300 import sss

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("rows,hq,hkv,dim,page,fresh,steps,seed", [(4, 8, 2, 128, 16, 3, 40, 1), (5, 4, 4, 64, 32, 5, 30, 2), (3, 16, 2, 64, 16, 40, 12, 3)])
def test_rows_cut_back(captured, rows, hq, hkv, dim, page, fresh, steps, seed):
    rng = np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    width = 500 // page + 1
    pages, t, most = rows * (width + 2), rows * fresh, width * page
    ints = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    table, new, past, lens, kv_len, parents = ints(rows, width).fill_(-1), ints(rows, width), ints(rows), ints(rows), ints(rows), ints(rows)
    src, dst, used, status, count = ints(rows), ints(rows), ints(1), ints(1), ints(1)
    free, new_tokens = torch.arange(pages, dtype=torch.int32, device=DEV), ints(rows).fill_(fresh)
    cu, positions, slots = ints(rows + 1), ints(t), ints(t)
    cache, buffer = sss.empty_kv_cache_q4(pages, page, hkv, dim), sss.empty_kv_cache(-(-t // 16), 16, hkv, dim)
    angle = torch.outer(torch.arange(most, device=DEV), 0.01 ** torch.linspace(0, 1, dim // 2, device=DEV))
    weight = torch.linspace(0.5, 1.5, dim, device=DEV)
    rope = sss.Rope(angle.cos(), angle.sin(), sss.ROPE_HALF, weight, weight)
    q, k, v = (torch.zeros((t, h * dim), device=DEV) for h in (hq, hkv, hkv))
    turned, out = torch.zeros((t, hq, dim), dtype=BF, device=DEV), torch.zeros((t, hq, dim), dtype=BF, device=DEV)
    need = sss.sss_attention_q4_workspace_bytes(t, hq, cache, rows, fresh, most, width)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None

    def step():
        sss.sss_page_fork(parents, past, page, free, table, new, lens, src, dst, used, dev_status=status)
        sss.sss_page_copy(cache, src, dst, dev_status=status)
        sss.sss_page_reclaim(new, lens, page, free, count, dev_status=status)
        sss.sss_page_plan(lens, new_tokens, page, free, new, cu, kv_len, positions, slots, used, dev_status=status)
        sss.sss_qk_norm_rope(q, k, v, rope, positions, buffer, q_out=turned, dev_status=status)
        sss.sss_kv_store_q4(buffer.k[:t], buffer.v[:t], cache, slots, dev_status=status)
        sss.sss_attention_q4(turned, cache, cu, kv_len, fresh, most, new, out=out, workspace=ws, dev_status=status)
        sss.sss_page_reclaim(new, kv_len, page, free, count, dev_status=status)
        table.copy_(new)

    graph = None
    if captured:
        step()  # (the kernels' first calls)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        table.fill_(-1)
        past.zero_()
        free.copy_(torch.arange(pages, dtype=torch.int32))
        status.zero_()
    seen = [[] for _ in range(rows)]  # per row: the numbers of its tokens
    keys, values = [], []
    for n in range(steps):
        choice = rng.integers(0, rows, rows) if n % 4 == 1 else np.arange(rows)
        parents.copy_(torch.from_numpy(choice.astype(np.int32)))
        past.copy_(torch.tensor([len(x) for x in seen], dtype=torch.int32))
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        step() if graph is None else graph.replay()
        torch.cuda.synchronize()
        assert int(status) == 0
        seen = [seen[p] + list(range(n * t + r * fresh, n * t + (r + 1) * fresh)) for r, p in enumerate(choice)]
        assert kv_len.tolist() == [len(x) for x in seen]
        # what was rotated, within its rounding; the cache then holds that in 4 bits
        at = positions.cpu().numpy()
        want = attn_plain.norm_rope(k.view(t, hkv, dim).cpu().numpy(), weight.cpu().numpy(), angle.cos().cpu().numpy(),
                                    angle.sin().cpu().numpy(), at, dim, True, 1e-6)
        err = np.abs(buffer.k[:t].cpu().double().numpy() - want[0])
        assert np.max(err / attn_plain.norm_rope_bound(*want, BF, dim)) <= 1.0
        assert at.tolist() == [x for s in seen for x in range(len(s) - fresh, len(s))]
        keys.append(buffer.k[:t].cpu().clone())
        values.append(buffer.v[:t].cpu().clone())
        if n % 3 == 2 or n == steps - 1:
            packed = [q4_plain.quantize(torch.cat(x).float().numpy()) for x in (keys, values)]
            kv = [len(x) for x in seen]
            w = q4_plain.attention(turned.cpu(), *[(q4_plain.values(u, s), s) for u, s, _ in packed], cu.tolist(), kv,
                                   lambda b: np.array(seen[b]), dim ** -0.5)
            bound = q4_plain.bound_many if fresh * hq // hkv > 64 else q4_plain.bound_rows
            assert np.max(np.abs(out.cpu().double().numpy() - w["out"]) / bound(w, BF, dim, max(kv))) <= 1.0
        # rejected tokens, and now and then a row back to anywhere
        for r in range(rows):
            cut = rng.integers(0, fresh + 1) if rng.random() < 0.8 else rng.integers(0, len(seen[r]) + 1)
            seen[r] = seen[r][:len(seen[r]) - cut]
        for r in range(rows):
            if len(seen[r]) + fresh > most - page:
                seen[r] = seen[r][:page + 3]
