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
