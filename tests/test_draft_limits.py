"""Numbers of sequences and groups next to 2^31, with which counters and sums of places in 32 bits would go past it, and scales next to the end of their range:
refused, no GPU is needed."""
import pytest

from paper_2510_11062_amd import api
from tests.test_draft_refusals import AT, EINVAL, EUNSUPPORTED, EWORKSPACE, call_plan, call_rules, plan_args, rules_args


@pytest.mark.parametrize("n_group", [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 1000])
def test_groups_of_a_plan(n_group):
    assert call_plan(plan_args(n_group=n_group, group_seq=1 << 52, prefix_len=1 << 53)) == EUNSUPPORTED


@pytest.mark.parametrize("over", [dict(n_seq=2 ** 31 - 1), dict(n_seq=2 ** 31 - 64), dict(n_group=2 ** 31 - 1), dict(n_group=2 ** 31 - 64)])
def test_sequences_and_groups_of_rules(over):
    assert call_rules(rules_args(**over)) == EUNSUPPORTED


@pytest.mark.parametrize("name", ["tree", "prefix"])
@pytest.mark.parametrize("scale,status", [(3e38, EINVAL), (2.4e38, EINVAL), (float("inf"), EINVAL), (float("nan"), EINVAL), (-1.0, EINVAL), (2.3e38, EWORKSPACE)])
def test_scales_whose_multiple_is_infinite(name, scale, status):
    """Exponents are scores times scale log2 e.  (A scale that is taken is refused for its workspace.)"""
    lib, C = api.load_library(), api.C
    kv = api._KV(1, 2, 64, 16, 100, 4, 8, 0, 0, *[next(AT) for _ in range(4)], None, None, None, None)
    q, out = api._Rows(next(AT), 256, 64), api._Rows(next(AT), 256, 64)
    if name == "tree":
        got = lib.at_grpo_tree_attention(C.byref(kv), 4, 4, C.byref(q), next(AT), scale, 8, C.byref(out), None, None, next(AT), 100, None)
    else:
        got = lib.at_grpo_prefix_attention(C.byref(kv), 4, 4, C.byref(q), scale, 1, 8, C.byref(out), None, None, next(AT), 100, None)
    assert got == status
