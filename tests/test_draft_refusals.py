"""What the calls on drafted tokens refuse on the host, before anything is launched: no GPU is needed, and the addresses hold nothing."""
import pytest

from paper_2510_11062_amd import api
from tests import test_rollout_abi

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


def rules_args(**over):
    f = {n: 0 for n, _ in api._SamplingRules._fields_}
    f.update(dtype=1, out_dtype=1, V=1000, n_seq=4, n_group=1, max_tokens=50, max_prompt=60, n_bias=5, n_mask=2)
    f.update({n: next(AT) for n, t in api._SamplingRules._fields_ if t is api.C.c_void_p})
    f.update(n_rows=9, logits=next(AT), stride=1000, out=next(AT), out_stride=1000, lse=next(AT), best=next(AT), workspace=next(AT), bytes=1 << 20)
    f.update(over)
    return f


def call_rules(f):
    r = api._SamplingRules(*(f[n] for n, _ in api._SamplingRules._fields_))
    return api.load_library().at_grpo_logit_rules(api.C.byref(r), f["n_rows"], f["logits"], f["stride"], f["out"], f["out_stride"], f["lse"], f["best"], None,
                                                  f["workspace"], f["bytes"], None)


@pytest.mark.parametrize("over,status", [
    (dict(n_rows=-1), EINVAL), (dict(V=0), EINVAL), (dict(n_seq=-1), EINVAL), (dict(n_group=-1), EINVAL), (dict(max_tokens=-1), EINVAL), (dict(max_prompt=-1), EINVAL),
    (dict(n_bias=-1), EINVAL), (dict(n_mask=-1), EINVAL), (dict(dtype=2), EUNSUPPORTED), (dict(dtype=0), EUNSUPPORTED), (dict(out_dtype=2), EUNSUPPORTED),
    (dict(V=2 ** 31 - 1), EUNSUPPORTED), (dict(max_tokens=2 ** 31 - 1), EUNSUPPORTED), (dict(max_prompt=2 ** 31 - 1), EUNSUPPORTED),
    (dict(n_bias=2 ** 31 - 1), EUNSUPPORTED), (dict(V=1 << 30, n_rows=1 << 20, stride=1 << 30, out_stride=1 << 30), EUNSUPPORTED),
    (dict(cu_q=None), EINVAL), (dict(logits=None), EINVAL), (dict(out=None, lse=None, best=None), EINVAL), (dict(stride=999), EINVAL), (dict(out_stride=999), EINVAL),
    (dict(length=None), EINVAL), (dict(group_seq=None), EINVAL), (dict(prompt_len=None), EINVAL), (dict(drafted=None), EINVAL), (dict(bias_token=None), EINVAL),
    (dict(bias=None), EINVAL), (dict(mask_row=None), EINVAL), (dict(logits=(1 << 51) + 1), EINVAL), (dict(out=(1 << 51) + 1), EINVAL),
    (dict(workspace=None), EWORKSPACE), (dict(bytes=16), EWORKSPACE), (dict(workspace=(1 << 51) + 8), EWORKSPACE)])
def test_rules(over, status):
    assert call_rules(rules_args(**over)) == status


@pytest.mark.parametrize("apart,stride,out_dtype", [(2, 1000, 1), (0, 1001, 1), (0, 1000, 0), (-2, 1000, 1), (17998, 1000, 1)])
def test_rules_outputs_that_meet_the_logits(apart, stride, out_dtype):
    f = rules_args(out_stride=stride, out_dtype=out_dtype)
    f["out"] = f["logits"] + apart
    assert call_rules(f) == EINVAL


def test_rules_of_no_rows():
    assert call_rules(rules_args(n_rows=0)) == 0
    r = api._SamplingRules(1, 1, 1000, 4)
    lib = api.load_library()
    assert lib.at_grpo_logit_rules_workspace_bytes(api.C.byref(r), -1) == 0 and lib.at_grpo_logit_rules_workspace_bytes(None, 5) == 0
    sizes = [lib.at_grpo_logit_rules_workspace_bytes(api.C.byref(r), n) for n in (0, 1, 100, 10 ** 6)]
    assert sizes == sorted(sizes) and sizes[0] > 0


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("g++", "-std=c++17")])
def test_struct_layout(tmp_path, monkeypatch, compiler, std):
    monkeypatch.setattr(test_rollout_abi, "MIRRORS", {"at_grpo_page_pool": api._PagePool, "at_grpo_sampling_rules": api._SamplingRules})
    test_rollout_abi.test_struct_layout(tmp_path, compiler, std)


def test_tree_attention():
    lib = api.load_library()
    kv = dict(dtype=1, Hk=2, D=64, page_size=16, n_pages=100, n_seq=4, max_pages=8, n_group=1, max_prefix_pages=9)
    ptr = {n: next(AT) for n in ("k", "v", "pages", "length", "cu_q", "group_seq", "prefix_len", "prefix_pages")}

    def call(ancestors=None, Hq=4, n_tok=9, scale=0.1, max_q=8, bytes=1 << 40, **over):
        sizes, ptrs = dict(kv, **{k: x for k, x in over.items() if k in kv}), dict(ptr, **{k: x for k, x in over.items() if k in ptr})
        c = api._KV(*sizes.values(), *ptrs.values())
        q, out = api._Rows(next(AT), 256, 64), api._Rows(next(AT), 256, 64)
        if over.get("in_place"):
            out = q
        return lib.at_grpo_tree_attention(api.C.byref(c), n_tok, Hq, api.C.byref(q), ancestors, scale, max_q, api.C.byref(out), None, None, next(AT), bytes, None)

    words = next(AT)
    assert call(None) == EINVAL and call(words, n_tok=0) == 0 and call(words, in_place=True) == EINVAL and call(words, bytes=100) == EWORKSPACE
    for over, status in ((dict(Hq=3), EINVAL), (dict(scale=0.0), EINVAL), (dict(max_q=0), EINVAL), (dict(k=None), EINVAL), (dict(length=None), EINVAL),
                         (dict(cu_q=None), EINVAL), (dict(prefix_pages=None), EINVAL), (dict(D=12), EUNSUPPORTED), (dict(D=264), EUNSUPPORTED), (dict(dtype=2), EUNSUPPORTED),
                         (dict(page_size=20), EUNSUPPORTED), (dict(n_tok=2 ** 31 - 1), EUNSUPPORTED)):
        assert call(words, **over) == status, over
    c = api._KV(*kv.values(), *[None] * 8)
    assert lib.at_grpo_tree_attention_workspace_bytes(api.C.byref(c), 9, 4, 8) > 0 and lib.at_grpo_tree_attention_workspace_bytes(api.C.byref(c), 9, 3, 8) == 0
