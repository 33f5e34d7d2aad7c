"""Attention of groups whose tokens are cut into parts of one step and longer ones, several to a CTA, against the plain form in 64 bits."""
import random

import pytest
import torch

from shared_cut import TWENTY, cut, one_step_ahead_of_another
from test_gpu_kv import Step
from test_gpu_kv_shared import shared_check, tt  # noqa: F401

pytestmark = pytest.mark.gpu


def run(tt, D, H, heads, prompts, seed):  # noqa: F811
    groups, before = [], []
    for i, (n, tokens) in enumerate(prompts):
        groups.append((len(before), len(before) + n, tokens))
        before += [tokens + (i + j) % 5 for j in range(n)]
    st = Step(seed, D, H, 64, before, [1] * len(before))
    shared_check(tt, st, heads, groups)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_twenty_prompts(tt, D):  # noqa: F811
    run(tt, D, 8, 32, TWENTY, 401)


@pytest.mark.parametrize("D,seed", [(64, 1), (128, 2), (128, 3), (64, 4)])
def test_prompts_that_leave_a_cta_one_step_ahead_of_another_part(tt, D, seed):  # noqa: F811
    ctas, rng = torch.cuda.get_device_properties(0).multi_processor_count, random.Random(seed)
    while True:
        H = rng.choice([1, 2, 4, 8])
        prompts = [(rng.randint(2, 4), 64 * rng.choice([2, 3, rng.randint(2, 30)])) for _ in range(rng.randint(2, 50))]
        if one_step_ahead_of_another(cut(D, H, 4, prompts, ctas)):
            break
    run(tt, D, H, 4 * H, prompts, 410 + seed)
