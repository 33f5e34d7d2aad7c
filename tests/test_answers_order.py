"""Which kernels read ahead of a wait of their own, and on what ground: the first kernel of the call has waited before it lets them start.  Read
from the source, as a run does not show it."""
import re

import test_launch_order_source as order

TEXT = dict(order.sources())


def test_the_first_kernel_waits_before_it_reads_or_releases():
    body = order.KERNELS["k_kv_prefix"][1]
    wait, release = body.index("pdl_wait();"), body.index("pdl_release();")
    assert wait < release
    for read in ("p.c.", "p.q", "p.g.", "p.seqs", "p.pieces", "make_plan", "part_of", "ldg", "tcgen05"):
        assert read not in body[:wait], read


def test_the_second_kernel_ends_behind_the_first_one():
    """It may read the call's operands, but nothing of the first kernel's, and its completion implies that one's."""
    body = order.KERNELS["k_kv_attend"][1]
    assert re.fullmatch(r"\s*if \(!SHARED\) \{\s*pdl_wait\(\);\s*pdl_release\(\);\s*\}\s*attend<D, NT, SHARED>\(p\);\s*if \(SHARED\) end_behind_prefix\(\);\s*\}", body)
    shared = TEXT["kv_shared.cuh"]
    assert re.search(r"void end_behind_prefix\(\) \{\s*pdl_release\(\);\s*pdl_wait\(\);\s*\}", shared)
    assert "p.pieces" in TEXT["kv_prefix.cu"] and "SharedSeq" not in TEXT["kv_attend.cu"].replace("reinterpret_cast<SharedSeq*>", "")


def test_the_third_kernel_reads_what_the_others_wrote_behind_its_wait():
    body = order.KERNELS["k_kv_join"][1]
    before = body[:body.index("pdl_wait();")]
    assert "sequence_of(p.c, r, lane, a, b)" in before  # operands of the call: row_start and no more
    for written in ("p.seqs", "p.owns", "p.own", "p.pieces", "p.out", "ldcg", "load_four"):
        assert written not in before, written
    lookup = TEXT["kv_common.cuh"]
    lookup = lookup[lookup.index("int sequence_of("):lookup.index("int block_of(")]
    assert set(re.findall(r"c\.(\w+)", lookup)) <= {"seqs", "row_start", "rows_of"}
    assert body.index("pdl_wait();") < body.index("pdl_release();")


def test_the_call_launches_them_in_this_order():
    text = TEXT["kv_attend.cu"]
    text = text[text.index("int tetra_kv_attend_shared("):]
    assert text.index("launch_prefix(") < text.index("launch_attend_all<true>(") < text.index("launch_join(")


def test_no_other_kernel_of_the_cache_and_of_tokens_reads_ahead_of_its_wait():
    for name in ("k_kv_append", "k_kv_append_at", "k_kv_append_blocks", "k_kv_read", "k_logprobs", "k_sample"):
        if name in order.KERNELS:
            body = order.KERNELS[name][1]
            before = body[:body.index("pdl_wait();")] if "pdl_wait();" in body else ""
            for read in ("sequence_of", "block_of", "c.record", "ldg", "load_row", "row_start", "lengths", "p.q", "p.k"):
                assert read not in before, (name, read)
