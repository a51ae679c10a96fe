"""The standard convolution's and linear layer's plan object on the host."""
import pytest


@pytest.mark.parametrize("make", [lambda wq: wq.DirectPlan(1, 8, 8, 64, 64, 64), lambda wq: wq.DirectPlan(16, 1, 1, 256, 64, 64, linear=True),
                                  lambda wq: wq.LinearPlan(16, 256, 64, 64)], ids=["conv", "linear", "linear_plan"])
def test_a_layout_in_hand_follows_the_plans_tuning(wq, make):
    """A caller that keeps plan.layout sees what wq_direct_plan_tune changes in it."""
    plan = make(wq)
    held = plan.layout
    for n in (1, 3 if held.taps == 9 else 4):
        plan.tune(n)
        assert held is plan.layout and held.splits == n and held.launch & 0xff == plan.launch[2]
