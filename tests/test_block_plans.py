"""The plans of layer normalisation and of the fully connected passes on tensors held in blocks, without a GPU: what they launch covers
the tensors and is within what a launch can be, whatever the sizes."""
import random

import pytest

FWD, BWD = 0, 1


def _sizes(seed, count, most):
    """Sizes over their logarithms, and those next to a power of two or at the ends."""
    g = random.Random(seed)
    ends = [1, 2, 3, 127, 128, 129, most - 1, most]
    return [g.choice(ends) if g.random() < 0.1 else max(1, min(most, round(most ** g.random()) + g.choice([-1, 0, 0, 1])))
            for _ in range(count)]


def test_filter_gradient_plans_cover_the_tensors(block_plans):
    for N, I, O, dtype in zip(_sizes(1, 4000, 1 << 14), _sizes(2, 4000, 1 << 15), _sizes(3, 4000, 1 << 15), [0, 1] * 2000):
        p = block_plans.kept_grad(N, I, O, dtype)
        if p == -2:
            assert N * -(-I // 128) * 128 >= 1 << 31 or N * O >= 1 << 31 or I * O >= 1 << 31
            continue
        assert p["blocks"] * 256 < 1 << 32
        if p["slices"]:
            assert N <= 16 * p["slices"] <= 128 and p["otiles"] * 128 >= O
            steps = -(-I // 64)
            assert (p["itiles"] - 1) * p["rows_per_split"] < steps <= p["itiles"] * p["rows_per_split"]
        else:
            assert p["otiles"] * p["tile"] >= O and p["itiles"] * p["tile"] >= I and p["splits"] * p["rows_per_split"] >= N
            assert p["rows_per_split"] % p["step"] == 0 and p["blocks"] >= p["itiles"] * p["otiles"] * p["splits"]
            assert p["bytes"] >= (p["splits"] * I * O * 4 if p["splits"] > 1 else 0)


def test_layer_norm_plans_cover_the_tensors(block_plans):
    for N, C, dtype in zip(_sizes(4, 4000, (1 << 31) - 1), _sizes(5, 4000, 1 << 27), [0, 1] * 2000):
        for op in (FWD, BWD):
            p = block_plans.layer_norm(op, N, C, dtype)
            if p == -2:
                assert N * C >= 1 << 40
                continue
            assert p["blocks"] * p["threads"] < 1 << 32 and p["threads"] <= 1024 and p["lds"] <= 160 * 1024
            assert p["wide"] or p["waves"] * p["regs"] * 64 * (8 if dtype else 4) >= C
            if p["apart"]:
                assert p["part_rows"] * p["rows_per_part"] >= N > (p["part_rows"] - 1) * p["rows_per_part"]
                assert p["part_rows"] * -(-C // 64) * 1024 < 1 << 32
            assert op == FWD or p["join_blocks"] * 1024 < 1 << 32
            if op == BWD and not p["wide"]:
                # a thread's columns are summed over at most 256 rows in fp32
                assert p["columns"] or p["apart"] or -(-N // (p["row_blocks"] * p["groups"])) <= 256


def test_the_columns_of_the_longest_rows_are_joined_in_one_launch(block_plans):
    for N in (0, 1, 700, 8191):
        for C in (1 << 27, (1 << 27) - 63, (1 << 27) - 64):
            assert block_plans.layer_norm(BWD, N, C, 0)["join_blocks"] * 1024 < 1 << 32


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("N,I,O", [(1, 1, (1 << 31) - 1), (1, 1, (1 << 31) - 127), (1, 1, (1 << 31) - 128), (1, (1 << 31) - 128, 1),
                                   (1, (1 << 31) - 255, 1), (0, (1 << 31) - 1, 1), (0, 1, (1 << 31) - 1), (0, 46340, 46340),
                                   (1, 3, (1 << 30) // 3 * 2), (2, 1, (1 << 30) - 1), (128, 1, (1 << 24) - 1), (129, 7, (1 << 24) - 200000)])
def test_filter_gradients_of_the_longest_tensors(block_plans, N, I, O, dtype):
    """Fewer than 2^31 elements each, as the header has it: positive counts, that a launch can hold, and nothing past the ends."""
    p = block_plans.kept_grad(N, I, O, dtype)
    assert min(p.values()) >= 0 and p["blocks"] * 256 < 1 << 32
    if N == 0:
        assert p["blocks"] == 0
    elif N <= 128:
        assert p["otiles"] * p["itiles"] == p["blocks"] and p["otiles"] * 128 >= p["outputs"]
        assert p["outputs"] == O or p["outputs"] % 128 == 0
        assert p["itiles"] * p["rows_per_split"] * 64 >= I
    else:
        assert p["otiles"] * p["tile"] >= O == p["outputs"] and p["itiles"] * p["tile"] >= I
