"""What the kernel of log probabilities must keep to, read from its source because a run does not show it."""
import re

import test_launch_order_source as order

TEXT = dict(order.sources())["logprobs.cu"]


def test_what_other_ctas_add_to_is_zero_before_they_are_told_to():
    """A cluster's CTAs write to the first one's memory behind a barrier at which it arrives early: nothing that they add to is set behind
    that, and nothing that they store is."""
    run = TEXT[TEXT.index("void lp_run("):]
    run = run[:run.index("__global__")]
    arrive = run.index("barrier_arrive")
    remote = set(re.findall(r"to->(\w+)", run))
    assert remote == {"count", "sums", "gathered"}
    assert re.findall(r"atomicAdd\(&to->(\w+)", run) == ["count"]
    zero = [m.start() for m in re.finditer(r"sm\.count\[[^\]]*\] = ", run)]
    assert len(zero) == 1 and zero[0] < arrive
    for name in ("sums", "gathered"):
        assert not re.search(r"sm\.%s(\[[^\]]*\])? = " % name, run), name
