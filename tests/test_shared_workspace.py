"""The workspace of the attention of groups, without a GPU: more rows, groups or query heads take no less, wherever its parts' bounds change."""
import pytest

from test_step_host import tt  # noqa: F401


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("kv", [1, 8])
def test_more_takes_no_less(tt, D, kv):  # noqa: F811
    size = tt.lib().tetra_kv_shared_workspace_bytes
    per = sorted({*range(1, 65), 96, 127, 128, 129, 255, 256, 512, 1024, 4096 // kv} & set(range(1, 4096 // kv + 1)))
    for groups in (0, 1, 40, 1024):
        last = None
        for rows in sorted({0, 1, 2, 7, 63, 64, 211, 1000, 1023, 1024, 1025, 2047, 2048, 2049, 8191, 8192, 8193, 65535, 65536} | {8192 // g + d for g in per for d in (-1, 0, 1)} - {-1}):
            made = [size(D, rows, kv * g, kv, groups) for g in per]
            assert all(a <= b for a, b in zip(made, made[1:])), (rows, groups)
            assert last is None or all(a <= b for a, b in zip(last, made)), (rows, groups)
            last = made
    for rows in (1, 211, 1024, 65536):
        made = [size(D, rows, 4 * kv, kv, g) for g in range(1025)]
        assert made == sorted(made)


def test_there_is_room_for_every_run(tt):  # noqa: F811
    """Runs of own tokens: each item of eight columns has one, and the warps of a grid of 384 CTAs one each beside that; a run is eight
    columns of D sums, a reference and a denominator."""
    size = tt.lib().tetra_kv_shared_workspace_bytes
    for D in (64, 128, 256):
        for kv in (1, 8):
            for group in (1, 2, 3, 5, 7, 8, 13, 64):
                for rows in (1, 100, 8192 // group):
                    # the most items that rows in up to 1024 sequences, eight columns each on average, may have
                    items = kv * max(n * -(-(rows // n) * group // 8) + -(-(rows % n) * group // 8) for n in {1, min(rows, 1024)})
                    assert size(D, rows, kv * group, kv, 1) >= (items + 8 * 384) * 8 * (D + 2) * 4
