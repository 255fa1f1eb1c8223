"""Order of the synchronising instructions in the 4-bit cache's and the shared pages'
kernels, read from their source: what a run cannot show, because it comes out right by
timing."""
import re

import pytest

from test_kernel_order import kernel_text


@pytest.mark.parametrize("file,name,reads", [
    ("kv_q4.cu", "kv_store_q4_kernel", ("a.slots[", "x[u].load(")), ("kv_q4.cu", "kv_fetch_q4_kernel", ("a.slots[", "s.table +", "s.kv_len[")),
    ("attn_rows_q4.cu", "attn_rows_q4_kernel", ("attn_tile(", "page = entry(")),
    ("page_share.cu", "page_fork_kernel", ("a.parents[", "a.past[", "a.table")), ("page_share.cu", "page_map_kernel", ("a.table", "held_entries(")),
    ("page_share.cu", "page_copy_kernel", ("a.src[", "a.dst[")),
])
def test_the_next_kernel_starts_only_behind_the_wait(file, name, reads):
    # (test_kernel_order.py says why)
    body = kernel_text(file, name)
    wait = body.index("griddepcontrol.wait")
    assert wait < body.index("griddepcontrol.launch_dependents")
    assert "return;" not in body[:wait]
    for read in reads:
        if read in body[:wait]:  # as part of a function that is called later
            assert "[&]" in body[:body.index(read)], read


def test_no_cta_leaves_while_a_peer_may_store_into_it():
    # as of the attention over 16-bit values (test_attention_order.py)
    body = kernel_text("attn_rows_q4.cu", "attn_rows_q4_kernel")
    arrives = [m.start() for m in re.finditer(r"barrier\.cluster\.arrive", body)]
    waits = [m.start() for m in re.finditer(r"barrier\.cluster\.wait", body)]
    stores = [m.start() for m in re.finditer(r"peer_store\(", body)]
    assert len(arrives) == 2 and len(stores) == 2
    assert arrives[0] < waits[1] < stores[0]
    assert stores[1] < arrives[1] < body.index("mbar_wait(&arrived", arrives[1]) < waits[-1]
    assert "return" not in body[arrives[1]:]
    assert "__all_sync(0xffffffffu, mbar_wait(&arrived" in body


def test_a_stage_is_read_before_it_is_filled_again():
    body = kernel_text("attn_rows_q4.cu", "attn_rows_q4_kernel")
    loop = body.index("for (int s = 0; s < mine; ++s) {")
    wait, again = body.index("mbar_wait(&full[warp][stage]", loop), body.index("issue(s + kStages, stage)", loop)
    last_read = max(body.rindex(x, loop, again) for x in ("lds(w, v)", "lds(vw[e][0], v)"))
    assert wait < last_read < body.index("__syncwarp();", last_read) < again
    # and the ring serves the join only when every copy has landed
    after = body.index("if (!waited)", again)
    assert body.index("mbar_wait(&full[warp][stage]", after) < body.index("float* part", after)


def test_the_map_outlives_its_readers():
    # every CTA arrives behind its last look at a peer's map before any leaves
    body = kernel_text("page_share.cu", "page_map_kernel")
    assert body.rindex("peer_word(") < body.rindex("cluster_meet()")
    assert "return" not in re.sub(r"const auto \w+ = \[&\].*?\n  };", "", body, flags=re.S)
    # the map's own bits are set, then joined slice by slice, then read whole: a wait between each two
    meets = [m.start() for m in re.finditer(r"cluster_meet\(\)", body)]
    looks = [m.start() for m in re.finditer(r"peer_word\(", body)]
    assert body.index("atomicOr(&map") < meets[0] < looks[0] < meets[1] < looks[1] < meets[2]
