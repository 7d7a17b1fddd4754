"""Numbers of sequences and groups next to 2^31, with which counters and sums of places in 32 bits would go past it: refused, no GPU is needed."""
import pytest

from tests.test_draft_refusals import EUNSUPPORTED, call_plan, call_rules, plan_args, rules_args


@pytest.mark.parametrize("n_group", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 1000])
def test_groups_of_a_plan(n_group):
    assert call_plan(plan_args(n_group=n_group, group_seq=1 << 52, prefix_len=1 << 53)) == EUNSUPPORTED


@pytest.mark.parametrize("over", [dict(n_seq=2 ** 31 - 1), dict(n_seq=2 ** 31 - 64), dict(n_group=2 ** 31 - 1), dict(n_group=2 ** 31 - 64)])
def test_sequences_and_groups_of_rules(over):
    assert call_rules(rules_args(**over)) == EUNSUPPORTED
