"""The barriers of the attention of many rows (attn_prompt.cu) on a model of its
roles, run in many orders: no role waits for ever, and none finds a barrier two
phases further than it looks (a wait tells phases apart by their parity alone)."""
import random

import pytest

from test_gemm_pipeline import Bar, finishes
from test_kernel_order import kernel_text


def roles(items, stages, keys_seen=True):
    """Generators of scheduler, producers (of queries and keys, and of values), issuer,
    tensor core, four warps that look through values, and 2 x 2 softmax warps (of 2 x 4) over items (n0, n1) of key
    tiles.  keys_seen: a stage of keys is given back by the issuer and by the warp
    that sees every key tile, not by the issuer alone."""
    pair = lambda n: [Bar(n), Bar(n)]  # noqa: E731
    full_q, empty_q, full_s, full_p, done, free_o = pair(1), pair(1), pair(1), pair(2), pair(1), pair(2)
    full_w, empty_w = pair(1), pair(11)
    ring = lambda n: [Bar(n) for _ in range(stages)]  # noqa: E731
    full_k, empty_k, full_v, seen, empty_v = ring(1), ring(2 if keys_seen else 1), ring(1), ring(4), ring(1)
    queue, works = [], [None, None]
    meet = Bar(4)

    def at(c):
        return c % stages, c // stages & 1

    def take(i):
        yield lambda: full_w[i & 1].passed(i >> 1 & 1)

    def scheduler():
        for i, n in enumerate(list(items) + [None]):
            yield lambda: empty_w[i & 1].passed(i >> 1 & 1 ^ 1)
            works[i & 1] = n
            full_w[i & 1].arrive()

    def copy(bar):  # a TMA copy: lands some time later
        flying.append(bar)

    flying = []

    def memory():
        while True:
            yield lambda: flying
            bar = flying.pop(rng.randrange(len(flying)))
            if bar is None:
                return
            bar.arrive()

    rng = random.Random(1)

    ended = []

    def producer(values):
        c, q = 0, [0, 0]
        i = 0
        while True:
            yield from take(i)
            n = works[i & 1]
            empty_w[i & 1].arrive()
            if n is None:
                yield lambda: not flying
                ended.append(values)
                if len(ended) == 2:
                    flying.append(None)
                return
            for j in range(max(n)):
                st, ph = at(c)
                yield lambda: (empty_v if values else empty_k)[st].passed(ph ^ 1)
                copy((full_v if values else full_k)[st])
                if j == 0 and not values:
                    for s in range(2):
                        if n[s]:
                            yield lambda: empty_q[s].passed(q[s] & 1 ^ 1)
                            copy(full_q[s])
                            q[s] += 1
                c += 1
            i += 1

    def issuer():
        c, q, p, o = 0, [0, 0], [0, 0], [1, 1]
        i = 0
        while True:
            yield from take(i)
            n = works[i & 1]
            empty_w[i & 1].arrive()
            i += 1
            if n is None:
                queue.append(None)
                return
            if max(n) == 0:
                continue
            st, ph = at(c)
            yield lambda: full_k[st].passed(ph)
            for s in range(2):
                if n[s]:
                    yield lambda: full_q[s].passed(q[s])
                    q[s] ^= 1
                    queue.append([full_s[s]] + ([empty_q[s]] if n[s] == 1 else []))
            queue.append([empty_k[st]])
            for s in range(2):
                if n[s]:
                    yield lambda: free_o[s].passed(o[s])
                    o[s] ^= 1
            for j in range(max(n)):
                st, ph = at(c)
                c += 1
                st1, ph1 = at(c)
                yield lambda: seen[st].passed(ph)
                for s in range(2):
                    if j >= n[s]:
                        continue
                    yield lambda: full_p[s].passed(p[s])
                    p[s] ^= 1
                    if j + 1 == n[s]:
                        queue.append([done[s]])
                    if j + 1 < n[s]:
                        queue.append([full_s[s]])
                    if j + 2 == n[s]:
                        queue.append([empty_q[s]])
                queue.append([empty_v[st]])
                if j + 1 < max(n):
                    queue.append([empty_k[st1]])

    def tensor_core():
        k = 0
        while True:
            yield lambda: k < len(queue)
            if queue[k] is None:
                return
            for b in queue[k]:
                b.arrive()
            k += 1

    def looker(wp):
        c = m = 0
        i = 0
        while True:
            yield from take(i)
            n = works[i & 1]
            empty_w[i & 1].arrive()
            i += 1
            for _ in range(1 if n is None else 3):
                meet.arrive()
                yield lambda: meet.passed(m)
                m ^= 1
            if n is None:
                return
            for j in range(max(n)):
                st, ph = at(c)
                c += 1
                st1, ph1 = at(c)
                yield lambda: full_v[st].passed(ph)
                if wp == 0:
                    if j == 0:
                        yield lambda: full_k[st].passed(ph)
                        if keys_seen:
                            empty_k[st].arrive()
                    if j + 1 < max(n):
                        yield lambda: full_k[st1].passed(ph1)
                        if keys_seen:
                            empty_k[st1].arrive()
                seen[st].arrive()

    def softmax(s):
        sp = dp = 0
        i = 0
        yield from take(0)
        after = works[0]
        while True:
            n = after
            if n is None:
                return
            for j in range(n[s]):
                yield lambda: full_s[s].passed(sp)
                sp ^= 1
                full_p[s].arrive()
            yield from take(i + 1)
            after = works[i + 1 & 1]
            if n[s]:
                yield lambda: done[s].passed(dp)
                dp ^= 1
                free_o[s].arrive()
            empty_w[i & 1].arrive()
            i += 1

    return ([scheduler(), producer(False), producer(True), issuer(), tensor_core(), memory()] + [looker(i) for i in range(4)]
            + [softmax(s) for s in (0, 0, 1, 1)])


ITEMS = [
    [(1, 1)] * 8, [(2, 2)] * 7, [(3, 4), (1, 1), (0, 2), (1, 0), (5, 5), (0, 0), (2, 3)],
    [(0, 0)] * 5 + [(1, 2), (0, 1)] + [(0, 0)] * 3 + [(4, 4)], [(1, 0), (0, 0), (2, 0), (1, 1), (6, 6)], [(16, 16), (1, 1), (8, 9)],
]


def all_finish(items, stages, keys_seen):
    rng = random.Random(str((items, stages)))
    for i in range(150):
        pick = rng.choice
        if i % 2:
            order = list(range(14))
            rng.shuffle(order)
            pick = lambda ready: min(ready, key=order.index)  # noqa: E731
        if not finishes(roles(items, stages, keys_seen), pick):
            return False
    return True


@pytest.mark.parametrize("stages", [2, 4])
@pytest.mark.parametrize("items", ITEMS)
def test_every_order_finishes(items, stages):
    assert all_finish(items, stages, True)


def test_the_model_sees_keys_that_overtake_the_warp_that_looks():
    assert not all_finish([(2, 2)] * 7, 2, False)


def test_the_kernel_gives_back_as_the_model_does():
    body = kernel_text("attn_prompt.cu", "attn_prompt_kernel")
    assert "mbar_init(&empty_k[s], 2);" in body
    assert body.count("mbar_arrive(&empty_k[") == 2 and body.count("umma_commit(&empty_k[") == 3
    assert body.count("mbar_wait(&full_k[") == 2 and body.count(" wait(&full_k[") == 1
