"""The kernels that the sizes of tests/quant_shapes.py are chosen for, by the plan's own rule (no GPU)."""
import pytest

import fp4_plan
import quant_shapes as shapes

pytestmark = pytest.mark.skipif(fp4_plan._program() is None, reason="no host C++ compiler or CUDA headers")


def dense(case):
    fmt, R, N, K = case
    return fp4_plan.plan(fmt, R, N, K)


def experts(case, tail=3):
    fmt, counts, N, K = case
    return fp4_plan.plan(fmt, sum(counts) + tail, N, K, len(counts))


@pytest.mark.parametrize("cases, slots", [(shapes.THREE_SLOTS, 3), (shapes.FIVE_SLOTS, 5)])
def test_odd_rings_are_gone_through_again(cases, slots):
    plans = [experts(c) for c in cases]
    assert all(not p.pair and p.splits == 1 and p.stages == slots and p.depth > 2 * slots for p in plans), plans
    for fmt in shapes.FORMATS:  # both ways of the scale bytes
        assert {p.raw for c, p in zip(cases, plans) if c[0] == fmt} == {False, True}


def test_odd_rings_of_dense_products():
    plans = [dense(c) for c in shapes.THREE_SLOTS_DENSE]
    assert all(not p.pair and p.splits == 1 and p.stages == 3 and p.depth > 3 for p in plans), plans
    assert {p.raw for p in plans} == {False, True}


def test_experts_of_the_pair_kernel():
    for c in shapes.PAIR_EXPERTS:
        p = experts(c, 0)
        assert p.pair and p.units > 2 * fp4_plan.SMS // 2, p


def test_tall_tiles_three_and_more_of_a_pair():
    plans = [dense(c) for c in shapes.TALL]
    assert all(p.pair and p.tile_tokens > 224 and p.units > 2 * (fp4_plan.SMS // 2) for p in plans), plans
    assert any(p.units > 3 * (fp4_plan.SMS // 2) for p in plans)
    assert {(c[0], p.slices) for c, p in zip(shapes.TALL, plans)} == {(0, 1), (1, 1), (1, 2)}
    assert {p.tile_tokens for p in plans} == {240, 256}


def test_tall_tiles_before_a_short_one():
    for c in shapes.TALL_AND_SHORT:
        p = dense(c)
        assert p.pair and p.tile_tokens > 224 and p.units > fp4_plan.SMS // 2 and 0 < c[1] % p.tile_tokens <= 32, p


def test_long_sums_in_one_part():
    for c in shapes.LONG:
        p = dense(c)
        assert p.splits == 1, p
