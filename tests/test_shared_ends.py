"""What the first kernel of the attention of groups must keep to when a wait of it runs out, read from the source because no run may show it."""
import re

import test_launch_order_source as order


def test_no_copy_is_in_flight_when_a_cta_ends():
    """The warp that copies waits for the last copies into each stage, whether it gave up itself or another warp did."""
    body = order.KERNELS["k_kv_prefix"][1]
    copies = body[body.index("if (warp == kPreCopyWarp) {"):body.index("} else if (warp >= kPreConvertAt")]
    wait = re.search(r"int none = 0;\s*for \(uint32_t back = 0; back < stages && back < issued; \+\+back\) \{.*?bar_wait\(smem_u32\(raw_full \+ --stage\), turn & 1u, &none\);", copies, re.S)
    assert wait
    before = copies[:wait.start()]
    assert before.count("{") - before.count("}") == 1  # in no branch but the warp's own


def test_every_wait_has_a_limit():
    text = dict(order.sources())["kv_prefix.cu"]
    assert text.count("mbarrier.try_wait") == 1 and "i < kPreTries" in text[text.index("bool bar_wait("):text.index("mbarrier.try_wait")]
