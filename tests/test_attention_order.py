"""Order of the synchronising instructions in the attention's kernels, read from their
source: what a run cannot show, because it comes out right by timing."""
import re

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
