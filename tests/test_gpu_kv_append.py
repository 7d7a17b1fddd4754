"""Appending normed and rotated keys, values and queries to a paged cache, against the oracle and, where the arithmetic is that of the
rotation call, against that call bit for bit."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as oracle
from paper_2510_11062_amd import api
from tests.rollout_case import Paged, assert_within, host64, i32, rounded, to_dev
from tests.test_gpu_qk_norm_rope import forward_bound

# dtype, Hq, Hk, D, rot, interleaved, page, lengths, new (None: one each), group sizes, prefixes
CASES = [
    ("bf16", 4, 2, 128, 128, False, 16, [1, 16, 17, 33], None, [4], [197]),
    ("f32", 2, 2, 64, 32, True, 8, [8, 9, 1], None, [1, 2], [0, 16]),
    ("bf16", 3, 1, 80, 20, False, 16, [5, 40, 0, 16], [5, 3, 0, 16], [2, 0, 1], [7, 3, 16]),      # the last sequence has no prefix
    ("bf16", 0, 2, 256, 256, False, 32, [70], [70], [], []),                                       # no queries
    ("f32", 8, 8, 8, 8, False, 64, [1, 2, 3], None, [], []),
    ("bf16", 16, 8, 128, 96, True, 64, [300, 1, 129], [300, 1, 64], [], []),
    ("bf16", 2, 1, 64, 64, False, 16, [3] * 200, None, [1] * 150, [5] * 150),                      # more groups than lanes
    ("f32", 2, 1, 64, 64, False, 16, [2] * 5000, [1, 0] * 2500, [50] * 90, list(range(90))),
]


def case(dev, spec, seed=0, norm=True):
    dtype, Hq, Hk, D, rot, inter, page, length, new, size, prefix = spec
    p = Paged(dtype, Hk, D, page, length, new, size, prefix, seed)
    most = int((p.before + p.length).max())
    c = dict(table=np.float64(np.float32(oracle.rope_table(most, rot, 1e4))))
    for name, h in (("q", Hq), ("k", Hk), ("v", Hk)):
        c[name] = rounded(p.rs.normal(size=(p.n_tok, h, D)) * 2, p.dtype)
    for name in ("q_weight", "k_weight"):
        c[name] = rounded(1 + 0.3 * p.rs.normal(size=D), p.dtype) if norm else None
    dv = {m: None if v is None else to_dev(v, torch.float32 if m == "table" else p.dtype, dev) for m, v in c.items()}
    if not Hq:
        dv["q"] = None
    return p, c, dv


def append(kv, dv, inter, **kw):
    return api.at_grpo_kv_append(kv, dv["q"], dv["k"], dv["v"], dv["table"], dv["q_weight"], dv["k_weight"], eps=1e-5, interleaved=inter, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("spec", CASES, ids=lambda s: f"{s[0]}-{s[1]}-{s[2]}-{s[3]}-page{s[6]}-{len(s[7])}")
def test_cache_and_queries(gpu_device, spec):
    p, c, dv = case(gpu_device, spec)
    inter, n = spec[5], p.n_tok
    kv = p.device(gpu_device)
    word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
    out = append(kv, dv, inter, data_error=word)
    # as the rotation call computes them, bit for bit
    position = oracle.append(p.k, p.v, p.pages, p.length, p.new, p.before, c["k"], c["v"])[2]
    rot = api.at_grpo_qk_norm_rope(dv["q"], dv["k"], dv["table"], i32(position, gpu_device), dv["q_weight"], dv["k_weight"], eps=1e-5, interleaved=inter)
    assert int(word) == 0
    k64 = host64(rot["k"])
    want_k, want_v, _ = oracle.append(p.k, p.v, p.pages, p.length, p.new, p.before, k64, c["v"])
    assert np.array_equal(host64(kv.cache_k), want_k, equal_nan=True) and np.array_equal(host64(kv.cache_v), want_v, equal_nan=True)
    if dv["q"] is None:
        assert out["q"] is None
    else:
        assert torch.equal(out["q"], rot["q"])
    if n <= 1000:
        args = c["k_weight"], c["table"], position
        ref = oracle.norm_rope(c["k"], *args, 1e-5, inter)
        assert_within(k64, ref, forward_bound(c["k"], *args, inter, ref, p.dtype), "k")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_norm_or_rotation_and_in_place(gpu_device, dtype):
    spec = (dtype, 4, 2, 128, 128, False, 16, [5, 40, 16], [5, 3, 1], [3], [9])
    p, c, dv = case(gpu_device, spec, norm=False)
    dv["table"] = None
    fused = torch.cat([dv[m].reshape(p.n_tok, -1) for m in ("q", "k", "v")], 1)
    views = dict(q=fused[:, :512].view(-1, 4, 128), k=fused[:, 512:768].view(-1, 2, 128), v=fused[:, 768:].view(-1, 2, 128))
    kv = p.device(gpu_device)
    before = fused.clone()
    append(kv, {**dv, **views}, False, q_out=views["q"])
    want_k, want_v, _ = oracle.append(p.k, p.v, p.pages, p.length, p.new, p.before, c["k"], c["v"])
    assert np.array_equal(host64(kv.cache_k), want_k, equal_nan=True) and np.array_equal(host64(kv.cache_v), want_v, equal_nan=True)
    assert torch.equal(fused, before)


@pytest.mark.gpu
def test_values_keep_their_bits(gpu_device):
    """NaN payloads and signed zeros too."""
    p, c, dv = case(gpu_device, CASES[0])
    bits = torch.randint(-(1 << 15), 1 << 15, dv["v"].shape, dtype=torch.int16, device=gpu_device)
    kv = p.device(gpu_device)
    append(kv, {**dv, "v": bits.view(torch.bfloat16)}, False)
    for s in range(4):
        i = int(p.length[s]) - 1
        assert torch.equal(kv.cache_v[p.pages[s][i // 16], :, i % 16].view(torch.int16), bits[s])


@pytest.mark.gpu
def test_data_errors(gpu_device):
    spec = ("bf16", 4, 2, 64, 64, False, 16, [5, 40, 16, 9], [2, 3, 1, 4], [2, 2], [9, 20])
    p, c, dv = case(gpu_device, spec)
    good = p.device(gpu_device)
    ref = append(good, dv, False)["q"]

    def run(bits, lost, **over):
        """`lost`: tokens that are left out"""
        word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
        kv = p.device(gpu_device, **over)
        q = append(kv, {**dv, **({"table": over.pop("table")} if "table" in over else {})}, False, data_error=word)["q"]
        assert int(word) == bits
        want_k, want_v = p.device(gpu_device), None
        k0, v0 = want_k.cache_k, want_k.cache_v
        for t in range(p.n_tok):
            s = int(np.searchsorted(p.cu_q, t, side="right")) - 1
            i = int(p.length[s] - p.new[s] + t - p.cu_q[s])
            if t in lost:
                assert not q[t].any()
            else:
                assert torch.equal(q[t], ref[t])
                k0[p.pages[s][i // 16], :, i % 16] = good.cache_k[p.pages[s][i // 16], :, i % 16]
                v0[p.pages[s][i // 16], :, i % 16] = good.cache_v[p.pages[s][i // 16], :, i % 16]
        assert torch.equal(kv.cache_k.view(torch.int16), k0.view(torch.int16)) and torch.equal(kv.cache_v.view(torch.int16), v0.view(torch.int16))

    run(0, [])
    pages = p.pages.copy()
    pages[1, 2] = p.n_pages                        # places 32 .. of sequence 1: its new tokens 37, 38, 39
    run(32, [2, 3, 4], pages=i32(pages, gpu_device))
    pages[1, 2] = -1
    run(32, [2, 3, 4], pages=i32(pages, gpu_device))
    for wrong in (-1, 1 << 20, 3):                   # fewer tokens than new ones, or more than the table holds
        length = p.length.copy()
        length[3] = wrong
        run(8, [6, 7, 8, 9], length=i32(length, gpu_device))
    prefix = p.prefix.copy()
    prefix[1] = 1 << 20
    run(8, [5, 6, 7, 8, 9], prefix_len=i32(prefix, gpu_device))
    prefix[1] = -1
    run(8, [5, 6, 7, 8, 9], prefix_len=i32(prefix, gpu_device))
    cu = p.cu_q.copy()
    cu[-1] = 8                                      # the last two tokens belong to nobody: new tokens of sequence 3 are two
    word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
    q = append(p.device(gpu_device, cu_q=i32(cu, gpu_device)), dv, False, data_error=word)["q"]
    assert int(word) == 8 and not q[8:].any() and torch.equal(q[:6], ref[:6])


@pytest.mark.gpu
def test_position_behind_the_table(gpu_device):
    p, c, dv = case(gpu_device, CASES[0])
    word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
    kv = p.device(gpu_device)
    q = append(kv, {**dv, "table": dv["table"][:-1].contiguous()}, False, data_error=word)["q"]
    assert int(word) == 64 and not q[3].any() and q[:3].any()
    assert torch.isnan(kv.cache_k[p.pages[3][2], :, 0]).any() == torch.isnan(to_dev(p.k, p.dtype, gpu_device)[p.pages[3][2], :, 0]).any()


@pytest.mark.gpu
def test_cache_past_two_gibielements(gpu_device):
    """A page whose first element stands behind 2^31."""
    Hk, page, D = 8, 64, 128
    n_pages = (1 << 31) // (Hk * page * D) + 3
    cache = [torch.zeros(n_pages, Hk, page, D, dtype=torch.bfloat16, device=gpu_device) for _ in range(2)]
    kv = api.KVBatch(*cache, pages=i32([[n_pages - 1]], gpu_device), length=i32([7], gpu_device))
    k, v = (torch.randn(1, Hk, D, device=gpu_device).bfloat16() for _ in range(2))
    api.at_grpo_kv_append(kv, None, k, v, None)
    assert torch.equal(cache[0][-1, :, 6], k[0]) and torch.equal(cache[1][-1, :, 6], v[0])
    assert int(torch.count_nonzero(cache[0][:3])) == 0 and int(torch.count_nonzero(cache[0][-3:])) == int(torch.count_nonzero(k))


@pytest.mark.gpu
def test_no_tokens_and_refusals(gpu_device):
    p, c, dv = case(gpu_device, CASES[0])
    kv = p.device(gpu_device)
    none = {m: (v[:0] if m in ("q", "k", "v") else v) for m, v in dv.items()}
    with pytest.raises(api.AtGrpoError):                  # a token for every sequence
        append(kv, none, False)
    zero = p.device(gpu_device, cu_q=i32(np.zeros(5), gpu_device))
    assert append(zero, none, False)["q"].shape == (0, 4, 128)
    for change in (dict(k=dv["k"].float()), dict(v=dv["v"][:, :1]), dict(k=dv["k"][:3]), dict(q=dv["q"][..., :64].contiguous()), dict(k=dv["k"].cpu()),
                   dict(q_weight=dv["q_weight"].float()), dict(table=dv["table"][..., :1])):
        with pytest.raises(api.AtGrpoError):
            append(kv, {**dv, **change}, False)
    t = dict(cache_k=kv.cache_k, cache_v=kv.cache_v, pages=kv.pages, length=kv.length, group_seq=kv.group_seq, prefix_len=kv.prefix_len,
             prefix_pages=kv.prefix_pages)
    for change in (dict(cache_v=kv.cache_v.float()), dict(cache_k=kv.cache_k[0]), dict(pages=kv.pages[:2]), dict(length=kv.length.long()),
                   dict(cu_q=kv.length), dict(prefix_len=None), dict(prefix_pages=kv.prefix_pages[:0]), dict(pages=kv.pages.cpu()),
                   dict(cache_k=kv.cache_k.transpose(1, 2))):
        with pytest.raises(api.AtGrpoError):
            api.KVBatch(**{**t, **change})


def test_refusals_of_the_library_on_the_host():
    lib, C = api.load_library(), api.C
    r = C.byref(api._Rows(4096, 64, 64))
    L = api._NormRope(1, 64, 64, 0, 10, 1e-6, 4096, 4096, 4096)

    def call(n=4, hq=2, **kw):
        a = dict(dtype=1, Hk=2, D=64, page_size=16, n_pages=9, n_seq=4, max_pages=3, n_group=1, max_prefix_pages=2, k=4096, v=4096, pages=4096,
                 length=4096, cu_q=None, group_seq=4096, prefix_len=4096, prefix_pages=4096)
        a.update(kw)
        return lib.at_grpo_kv_append(C.byref(api._KV(*a.values())), C.byref(L), n, hq, r, r, r, r, None, None)

    for kw, status in [(dict(dtype=3), 2), (dict(dtype=0), 1), (dict(D=128), 1), (dict(D=60), 2), (dict(page_size=4), 2), (dict(page_size=24), 2),
                       (dict(page_size=1 << 17), 2), (dict(n_pages=0), 1), (dict(Hk=0), 1), (dict(n_seq=-1), 1), (dict(k=None), 1), (dict(v=4100), 1),
                       (dict(pages=None), 1), (dict(length=None), 1), (dict(group_seq=None), 1), (dict(prefix_len=None), 1),
                       (dict(prefix_pages=None), 1), (dict(n=3), 1), (dict(n=-1), 1), (dict(hq=-1), 1), (dict(max_pages=1 << 28), 2), (dict(k=4100), 1)]:
        assert call(**kw) == status, kw


@pytest.mark.gpu
@pytest.mark.parametrize("group_seq,lost", [([0, 3, 2], [2]), ([0, 2, 5], [2, 3]), ([-1, 2, 4], [0, 1]), ([3, 2, 4], [2]), ([0, 1 << 30, 4], [0, 1, 2, 3])])
def test_groups_that_fall_or_leave_their_range(gpu_device, group_seq, lost):
    """A sequence that the entries around it do not enclose has no prefix to go by: its tokens are left out, as those of no sequence are."""
    spec = ("bf16", 4, 2, 64, 64, False, 16, [5, 40, 16, 9], [2, 3, 1, 4], [2, 2], [9, 20])
    p, c, dv = case(gpu_device, spec)
    word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
    kv = p.device(gpu_device, group_seq=i32(group_seq, gpu_device))
    q = append(kv, dv, False, data_error=word)["q"]
    assert int(word) == 8
    empty = p.device(gpu_device)
    for s in range(4):
        mine = slice(int(p.cu_q[s]), int(p.cu_q[s + 1]))
        assert bool(q[mine].any()) == (s not in lost)
        for i in range(int(p.length[s] - p.new[s]), int(p.length[s])):
            at = p.pages[s][i // 16], slice(None), i % 16
            for got, before in ((kv.cache_k, empty.cache_k), (kv.cache_v, empty.cache_v)):
                assert torch.equal(got[at].view(torch.int16), before[at].view(torch.int16)) == (s in lost)


@pytest.mark.gpu
def test_more_tokens_than_a_launch_counts_threads(gpu_device):
    """A wavefront a token: 7 * 10^7 new tokens are more than 2^32 threads."""
    n, page = 70_000_000, 1024
    n_pages = -(-n // page)
    cache = [torch.zeros(n_pages, 1, page, 8, dtype=torch.bfloat16, device=gpu_device) for _ in range(2)]
    kv = api.KVBatch(*cache, pages=torch.arange(n_pages, dtype=torch.int32, device=gpu_device)[None], length=i32([n], gpu_device), cu_q=i32([0, n], gpu_device))
    k = (torch.arange(n, device=gpu_device) % 251 + 1).bfloat16()[:, None, None].expand(n, 1, 8).contiguous()
    api.at_grpo_kv_append(kv, None, k, -k, None)
    assert torch.equal(cache[0].view(-1, 8)[:n], k[:, 0]) and torch.equal(cache[1].view(-1, 8)[:n], -k[:, 0])
    assert not cache[0].view(-1, 8)[n:].any()
