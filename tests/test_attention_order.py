"""Order of the synchronising instructions in the attention's kernels, read from their
source: what a run cannot show, because it comes out right by timing."""
import re

import pytest

from test_kernel_order import kernel_text


def test_no_cta_leaves_while_a_peer_may_store_into_it():
    # the join of a cluster's splits: all have started before the first store, all
    # arrive behind their stores, and nobody leaves before all have: on an expired wait
    # neither, and then what is under way lands
    body = kernel_text("attn_rows.cu", "attn_rows_kernel")
    arrives = [m.start() for m in re.finditer(r"barrier\.cluster\.arrive", body)]
    waits = [m.start() for m in re.finditer(r"barrier\.cluster\.wait", body)]
    stores = [m.start() for m in re.finditer(r"peer_store\(", body)]
    assert len(arrives) == 2 and len(stores) == 2
    assert arrives[0] < waits[1] < stores[0]  # (waits[0] is that of a CTA without work)
    assert stores[1] < arrives[1] < body.index("mbar_wait(&arrived", arrives[1]) < waits[-1]
    assert "return" not in body[arrives[1]:]
    assert body.index("mbar_wait(&arrived", waits[-1]) > waits[-1]
    # each wait's outcome is the warp's: its lanes go on together
    assert "__all_sync(0xffffffffu, mbar_wait(&arrived" in body


@pytest.mark.parametrize("file,name", [
    ("page_plan.cu", "page_plan_kernel"), ("qk_norm_rope.cu", "qk_norm_rope_kernel"), ("attn_prompt.cu", "attn_prompt_kernel"),
    ("attn_rows.cu", "attn_rows_kernel"), ("attn_rows.cu", "attn_join_kernel"),
])
def test_the_next_kernel_starts_only_behind_the_wait(file, name):
    # as of the other kernels (test_kernel_order.py), and nobody leaves before it
    body = kernel_text(file, name)
    wait = body.index("griddepcontrol.wait")
    assert wait < body.index("griddepcontrol.launch_dependents")
    assert "return" not in body[:wait]
    for read in ("cu_q", "kv_len", "a.positions", "a.past", "maps.q,", "a.slots"):
        assert read not in body[:wait]
