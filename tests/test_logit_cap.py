"""parason_plan_set_logit_cap where no GPU is needed: what it refuses, and that
a cap leaves the plan's work as it is."""
import math

import numpy as np
import pytest

from paper_2608_24658_gb300 import _lib, build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import ParasonError, Plan


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


@pytest.mark.parametrize("bad", [-1.0, math.nan, math.inf, -math.inf, 2.0 ** -11, 2.0 ** 21, 1e-30])
def test_refused_caps(bad):
    tree = W.figure3_tree(values=False)
    with Plan.for_tree(tree, host_only=True) as plan:
        with pytest.raises(ParasonError) as e:
            plan.set_logit_cap(bad)
        assert e.value.status == _lib.EINVAL
    with pytest.raises(ParasonError):
        Plan.for_tree(tree, host_only=True, logit_cap=bad)
    assert _lib.load().parason_plan_set_logit_cap(None, 30.0) == _lib.EINVAL


def test_scale_that_a_cap_overflows():
    with Plan.for_tree(W.figure3_tree(values=False, sm_scale=3e38), host_only=True) as plan:
        plan.set_logit_cap(4.0)
        with pytest.raises(ParasonError) as e:
            plan.set_logit_cap(0.5)
        assert e.value.status == _lib.EINVAL


@pytest.mark.parametrize("good", [0.0, 2.0 ** -10, 1.0, 50.0, 2.0 ** 20])
def test_caps_leave_the_plan_as_it_is(good):
    tree = W.pair_fixture(values=False)
    with Plan.for_tree(tree, host_only=True) as a, Plan.for_tree(tree, host_only=True, logit_cap=good) as b:
        assert a.info() == b.info()
        for table in range(_lib.TABLE_SHARD_BRANCHES + 1):
            assert np.array_equal(a.export(table), b.export(table))
    with Plan.for_tree(tree, host_only=True, logit_cap=good, shard=(_lib.SHARD_KV_HEADS, 0, 2)) as p:
        p.set_logit_cap(0.0)
