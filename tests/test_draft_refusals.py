"""What the calls on drafted tokens refuse on the host, before anything is launched: no GPU is needed, and the addresses hold nothing."""
import pytest

from paper_2510_11062_amd import api

EINVAL, EUNSUPPORTED, EWORKSPACE = 1, 2, 3
AT = iter(range(1 << 40, 1 << 50, 1 << 30))      # addresses far from each other


def plan_args(**over):
    names = ("length", "keep", "add", "parent", "state", "length_out", "state_out", "cu_q", "seq", "position", "slot", "ancestors")
    a = {n: next(AT) for n in names}
    a.update(page_size=16, n_pages=100, n_seq=10, max_pages=8, n_group=2, pages=next(AT), ring=next(AT), group_seq=next(AT), prefix_len=next(AT), n_tok=20,
             data_error=next(AT), workspace=next(AT), bytes=1 << 20)
    a.update(over)
    return a


def call_plan(a):
    pool = api._PagePool(*(a[n] for n in ("page_size", "n_pages", "n_seq", "max_pages", "n_group", "pages", "ring", "group_seq", "prefix_len")))
    return api.load_library().at_grpo_kv_plan(api.C.byref(pool), a["n_tok"], *(a[n] for n in (
        "length", "keep", "add", "parent", "state", "length_out", "state_out", "cu_q", "seq", "position", "slot", "ancestors", "data_error", "workspace", "bytes")), None)


@pytest.mark.parametrize("over,status", [
    (dict(n_tok=-1), EINVAL), (dict(n_pages=0), EINVAL), (dict(n_seq=-1), EINVAL), (dict(max_pages=-1), EINVAL), (dict(n_group=-1), EINVAL),
    (dict(page_size=7), EUNSUPPORTED), (dict(page_size=24), EUNSUPPORTED), (dict(page_size=1 << 17), EUNSUPPORTED), (dict(max_pages=(1 << 26) + 1), EUNSUPPORTED),
    (dict(n_seq=1 << 20, max_pages=1 << 11), EUNSUPPORTED), (dict(n_tok=2 ** 31 - 1), EUNSUPPORTED),
    (dict(ring=None), EINVAL), (dict(state=None), EINVAL), (dict(state_out=None), EINVAL), (dict(cu_q=None), EINVAL), (dict(length=None), EINVAL),
    (dict(add=None), EINVAL), (dict(length_out=None), EINVAL), (dict(pages=None), EINVAL), (dict(group_seq=None), EINVAL), (dict(prefix_len=None), EINVAL),
    (dict(parent=None), EINVAL),      # with ancestors
    (dict(workspace=None), EWORKSPACE), (dict(bytes=64), EWORKSPACE), (dict(workspace=(1 << 51) + 8), EWORKSPACE)])
def test_plan(over, status):
    assert call_plan(plan_args(**over)) == status


@pytest.mark.parametrize("out,other,apart", [("length_out", "length", 4), ("length_out", "add", 0), ("length_out", "keep", 0), ("state_out", "state", 4), ("cu_q", "add", -40),
                                             ("seq", "position", 0), ("seq", "slot", 156), ("ancestors", "parent", 79), ("pages", "ring", 396), ("slot", "cu_q", 40),
                                             ("data_error", "state", 4), ("ring", "prefix_len", 4)])
def test_plan_outputs_that_meet_something(out, other, apart):
    a = plan_args()
    a[out] = a[other] + apart
    assert call_plan(a) == EINVAL


def test_plan_workspace():
    lib = api.load_library()
    assert lib.at_grpo_kv_plan_workspace_bytes(-1) == 0
    sizes = [lib.at_grpo_kv_plan_workspace_bytes(n) for n in (0, 1, 100, 5000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and sizes[-1] >= 8 << 20
