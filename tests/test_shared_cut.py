"""Parts of the tokens that groups share, without a GPU: which calls give a CTA two parts whose columns both slots share, the first of one
step (the second slot's weights have no work in it), and that no warp can be two parts ahead of another then."""
import re

import test_launch_order_source as order
from shared_cut import TWENTY, cut, one_step_ahead_of_another


def test_ordinary_prompts_have_parts_of_one_step_ahead_of_others():
    for D in (64, 128):
        parts = cut(D, 8, 4, TWENTY, 148)
        assert sum(map(len, parts)) == 288 and max(s for mine in parts for s, _ in mine) == 5
        assert len(one_step_ahead_of_another(parts)) == 28


def body():
    return order.KERNELS["k_kv_prefix"][1]


def test_queries_are_announced_by_all_and_not_before_the_last_ones_were_seen():
    text = body()
    assert re.search(r"bar_init\(smem_u32\(&q_ready\), 4 \* SLOTS\)", text) and re.search(r"bar_init\(smem_u32\(&q_seen\), SLOTS\)", text)
    # one arrival, by every warp of the weights and in every part, directly behind the wait for the part before
    assert len(re.findall(r"bar_arrive\(smem_u32\(&?q_ready", text)) == 1
    assert re.search(r"bar_wait\(smem_u32\(&q_seen\), \(q_parts - 1\) & 1u, gave_up\);.*?\+\+q_parts;\s*__syncwarp\(\);\s*if \(lane == 0\) bar_arrive\(smem_u32\(&q_ready\)\);", text, re.S)
    # and each slot's products say so once a part, behind their own wait
    assert len(re.findall(r"bar_arrive\(smem_u32\(&q_seen\)\)", text)) == 1
    assert re.search(r"bar_wait\(smem_u32\(&q_ready\), q_parts & 1u, gave_up\);\s*ok = __all_sync\(0xFFFFFFFFu, ok\);\s*if \(!ok\) break;\s*if \(lane == 0\) bar_arrive\(smem_u32\(&q_seen\)\);", text)
