"""Norm and rotation of queries and keys, forward and gradient, and the rotation tables, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as oracle
from paper_2510_11062_amd import api
from tests.rollout_case import DTYPES, U16, U32, assert_within, host64, i32, rounded, to_dev

# sum of at most 256 squares in a tree of lanes, a square root, a division and four products: 16 roundings at most
EPS32 = 16 * U32

# dtype, tokens, Hq, Hk, D, rot_dim, interleaved, normed (queries, keys)
SHAPES = [
    ("f32", 1, 1, 1, 64, 64, False, (True, True)),
    ("bf16", 1, 16, 8, 128, 128, False, (True, True)),
    ("bf16", 5, 3, 1, 128, 64, True, (True, True)),
    ("f32", 7, 4, 2, 128, 32, False, (True, False)),
    ("bf16", 9, 5, 5, 80, 20, False, (True, True)),       # pairs that no vector of four holds
    ("f32", 3, 2, 7, 80, 50, True, (False, True)),
    ("bf16", 4, 2, 2, 256, 192, False, (True, True)),
    ("f32", 6, 2, 1, 256, 256, True, (True, True)),
    ("bf16", 33, 2, 2, 8, 8, False, (True, True)),
    ("f32", 11, 3, 2, 96, 2, False, (True, True)),
    ("bf16", 6, 4, 2, 128, 0, False, (True, True)),        # nothing turns
    ("bf16", 5, 4, 2, 64, 64, False, (False, False)),      # nothing is normed
    ("bf16", 130, 9, 0, 128, 96, True, (True, False)),     # queries alone
    ("f32", 65, 0, 5, 64, 48, False, (False, True)),       # keys alone
    ("bf16", 1500, 1, 1, 64, 64, False, (True, True)),     # more tokens than workgroups of the gradient
]


def case(dev, dtype, n, Hq, Hk, D, rot, interleaved, normed, seed=0):
    rs = np.random.default_rng([seed, n, D, rot])
    dt = DTYPES[dtype]
    c = dict(position=rs.integers(0, 300, n), table=np.float64(np.float32(oracle.rope_table(300, rot, 10000.0))) if rot else None)
    for name, h, w in (("q", Hq, normed[0]), ("k", Hk, normed[1])):
        c[name] = rounded(rs.normal(size=(n, h, D)) * 2, dt) if h else None
        c["d" + name] = rounded(rs.normal(size=(n, h, D)), dt) if h else None
        c[name + "_weight"] = rounded(1 + 0.3 * rs.normal(size=D), dt) if w else None
    dv = {k: None if v is None else (i32(v, dev) if k == "position" else to_dev(v, torch.float32 if k == "table" else dt, dev)) for k, v in c.items()}
    return c, dv


def forward(dv, interleaved, **kw):
    return api.at_grpo_qk_norm_rope(dv["q"], dv["k"], dv["table"], dv["position"], dv["q_weight"], dv["k_weight"], eps=1e-5,
                                    interleaved=interleaved, **kw)


def backward(dv, interleaved, **kw):
    return api.at_grpo_qk_norm_rope_bwd(dv["dq"], dv["dk"], dv["q"], dv["k"], dv["table"], dv["position"], dv["q_weight"], dv["k_weight"],
                                        eps=1e-5, interleaved=interleaved, **kw)


def forward_bound(x, w, table, position, interleaved, ref, dtype):
    """Both elements of a pair go into each result, so the error goes by their sum."""
    mags = oracle.norm_rope(np.abs(x), w if w is None else np.abs(w), None, position, 1e-5, interleaved)
    both = mags.copy()
    if table is not None:
        for a, b in oracle.pairs(2 * table.shape[1], interleaved):
            both[..., a] = both[..., b] = mags[..., a] + mags[..., b]
    return EPS32 * both + (U16 * np.abs(ref) if dtype == torch.bfloat16 else 0)


def grad_bounds(dy, x, w, table, position, interleaved, ref, dtype):
    g = np.abs(dy)
    if table is not None:
        for a, b in oracle.pairs(2 * table.shape[1], interleaved):
            g[..., a] = g[..., b] = g[..., a] + g[..., b]
    if w is None:
        bx, bw = EPS32 * g, None
    else:
        size = np.sqrt((x ** 2).mean(-1, keepdims=True) + 1e-5)
        n = np.abs(x) / size
        gw = g * np.abs(w)
        bx = 3 * EPS32 * (gw + n * (gw * n).mean(-1, keepdims=True)) / size
        bw = 3 * EPS32 * (g * n).sum((0, 1)) + U32 * np.sqrt(x.shape[0] * x.shape[1]) * (g * n).sum((0, 1))
    return bx + (U16 * np.abs(ref) if dtype == torch.bfloat16 else 0), bw


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s[:7]))
def test_forward_and_gradient(gpu_device, shape):
    dtype, n, Hq, Hk, D, rot, inter, normed = shape
    c, dv = case(gpu_device, *shape)
    out, grad = forward(dv, inter), backward(dv, inter)
    torch.cuda.synchronize()
    for name in ("q", "k"):
        if c[name] is None:
            assert out[name] is None and grad["d" + name] is None
            continue
        args = c[name + "_weight"], c["table"], c["position"]
        ref = oracle.norm_rope(c[name], *args, 1e-5, inter)
        assert_within(host64(out[name]), ref, forward_bound(c[name], *args, inter, ref, DTYPES[dtype]), name)
        dx, dw = oracle.norm_rope_grad(c["d" + name], c[name], *args, 1e-5, inter)
        bx, bw = grad_bounds(c["d" + name], c[name], *args, inter, dx, DTYPES[dtype])
        assert_within(host64(grad["d" + name]), dx, bx, "d" + name)
        if dw is None:
            assert grad[f"d{name}_weight"] is None
        else:
            assert_within(host64(grad[f"d{name}_weight"]), dw, bw, f"d{name}_weight")


@pytest.mark.parametrize("inter,rot,normed", [(False, 16, True), (True, 12, True), (False, 10, True), (True, 16, False)])
def test_oracle_gradient_against_differences(inter, rot, normed):
    rs = np.random.default_rng(5)
    x, dy, w = rs.normal(size=(3, 2, 16)), rs.normal(size=(3, 2, 16)), (rs.normal(size=16) if normed else None)
    table, pos = oracle.rope_table(9, rot, 100.0, magnitude=1.2), rs.integers(0, 9, 3)
    f = lambda x, w: float((dy * oracle.norm_rope(x, w, table, pos, 1e-3, inter)).sum())
    dx, dw = oracle.norm_rope_grad(dy, x, w, table, pos, 1e-3, inter)
    h = 1e-5      # central differences: h^2 f''' / 6 and 1e-15 / h, both below 1e-9 here
    for at in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[at] = h
        assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - dx[at]) < 1e-7
    for d in range(16 if normed else 0):
        e = np.zeros(16)
        e[d] = h
        assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - dw[d]) < 1e-7


@pytest.mark.gpu
def test_gradient_against_differences_of_the_forward(gpu_device):
    """fp32, along random directions; the forward in fp32 limits a difference with step h to about 1e-6 / h of its terms."""
    c, dv = case(gpu_device, "f32", 5, 2, 1, 64, 32, False, (True, True))
    grad = backward(dv, False)
    rs = np.random.default_rng(2)
    h = 2.0 ** -6
    for name in ("q", "k", "q_weight", "k_weight"):
        e = to_dev(rs.normal(size=c[name].shape), torch.float32, gpu_device)

        def value(sign):
            o = forward({**dv, name: dv[name] + sign * h * e}, False)
            return sum(float((dv["d" + r].double() * o[r].double()).sum()) for r in ("q", "k"))

        slope = (value(1) - value(-1)) / (2 * h)
        terms = (grad["d" + name].double() * e.double()).flatten()
        # third-order term: h^2 / 6 times a third derivative of the order of the terms themselves (rows of size 2); rounding 2^-24 / h
        assert abs(slope - float(terms.sum())) < (h * h + 64 * U32 / h) * float(terms.abs().sum()) + 1e-3


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter,rot", [(False, 128), (True, 96), (False, 36)])
def test_strides_and_in_place(gpu_device, dtype, inter, rot):
    """Views of one projection's output, heads in front of tokens, and outputs that are the inputs: the same bits as dense rows."""
    c, dv = case(gpu_device, dtype, 21, 6, 2, 128, rot, inter, (True, True))
    ref, gref = forward(dv, inter), backward(dv, inter)
    n, D = 21, 128
    fused = torch.cat([dv["q"].reshape(n, -1), dv["k"].reshape(n, -1), dv["k"].reshape(n, -1)], 1)
    q, k = fused[:, :6 * D].view(n, 6, D), fused[:, 6 * D:8 * D].view(n, 2, D)
    heads_first = {m: dv[m].transpose(0, 1).contiguous().transpose(0, 1) for m in ("dq", "dk")}
    rest = fused[:, 8 * D:].clone()
    out = forward({**dv, "q": q, "k": k}, inter)
    g = backward({**dv, **heads_first, "q": q, "k": k}, inter)
    for m in ("q", "k"):
        assert torch.equal(out[m], ref[m]) and torch.equal(g["d" + m], gref["d" + m]) and torch.equal(g[f"d{m}_weight"], gref[f"d{m}_weight"])
    g = backward({**dv, **heads_first, "q": q, "k": k}, inter, dq=heads_first["dq"], dk=heads_first["dk"])
    assert torch.equal(heads_first["dq"], gref["dq"]) and torch.equal(heads_first["dk"], gref["dk"])
    forward({**dv, "q": q, "k": k}, inter, q_out=q, k_out=k)
    assert torch.equal(q, ref["q"]) and torch.equal(k, ref["k"]) and torch.equal(fused[:, 8 * D:], rest)


@pytest.mark.gpu
def test_positions_outside_the_table(gpu_device):
    c, dv = case(gpu_device, "bf16", 6, 4, 2, 128, 64, False, (True, True))
    ref, gref = forward(dv, False), backward(dv, False)
    position = dv["position"].clone()
    position[1], position[4] = 300, -1
    keep = torch.tensor([0, 2, 3, 5], device=gpu_device)
    word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
    out = forward({**dv, "position": position}, False, data_error=word)
    assert int(word) == 64
    g = backward({**dv, "position": position}, False, data_error=word)
    some = backward({**{m: (v[keep] if m in ("q", "k", "dq", "dk", "position") else v) for m, v in dv.items()}}, False)
    for m in ("q", "k"):
        assert torch.equal(out[m][keep], ref[m][keep]) and not out[m][[1, 4]].any()
        assert torch.equal(g["d" + m][keep], gref["d" + m][keep]) and not g["d" + m][[1, 4]].any()
        assert torch.allclose(g[f"d{m}_weight"], some[f"d{m}_weight"], rtol=1e-5, atol=1e-5)
    word.zero_()
    forward(dv, False, data_error=word)
    assert int(word) == 0


@pytest.mark.gpu
def test_rows_of_zeros_and_of_large_numbers(gpu_device):
    c, dv = case(gpu_device, "f32", 4, 2, 2, 64, 64, False, (True, True))
    dv["q"][0] = 0
    dv["k"][1] = 1e18       # squares of 1e36: their sum stays below the largest float
    out, g = forward(dv, False), backward(dv, False)
    assert not out["q"][0].any() and all(torch.isfinite(t).all() for t in (out["q"], out["k"], g["dq"], g["dk"], g["dq_weight"], g["dk_weight"]))
    c["q"][0], c["k"][1] = 0, np.float64(np.float32(1e18))
    ref = oracle.norm_rope(c["k"], c["k_weight"], c["table"], c["position"], 1e-5, False)
    assert_within(host64(out["k"]), ref, forward_bound(c["k"], c["k_weight"], c["table"], c["position"], False, ref, torch.float32), "k")


@pytest.mark.gpu
def test_no_tokens(gpu_device):
    c, dv = case(gpu_device, "bf16", 3, 2, 1, 64, 64, False, (True, True))
    none = {m: (v[:0] if m in ("q", "k", "dq", "dk", "position") else v) for m, v in dv.items()}
    assert forward(none, False)["q"].shape == (0, 2, 64)
    g = backward(none, False)
    assert not g["dq_weight"].any() and not g["dk_weight"].any()


@pytest.mark.gpu
@pytest.mark.parametrize("scaling", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                     dict(scaling="parts", factor=16.0, trained=2048.0, slow=1.0, fast=32.0, magnitude=1.27)])
def test_tables(gpu_device, scaling):
    ref = oracle.rope_table(5000, 96, 5e5, **scaling)
    got = host64(api.at_grpo_rope_table(5000, 96, 5e5, device=gpu_device, **scaling))
    # angles up to 5000 in 64 bits (error 5000 * 2^-52 a few times over), then one rounding to fp32
    assert_within(got, ref, U32 * np.abs(ref) + 1e-10, "table")
    far = host64(api.at_grpo_rope_table(1 << 20, 2, 10000.0, device=gpu_device))[-1, 0]
    assert abs(far[0] - np.cos((1 << 20) - 1)) < 1e-7 and abs(far[1] - np.sin((1 << 20) - 1)) < 1e-7


@pytest.mark.gpu
def test_refusals(gpu_device):
    c, dv = case(gpu_device, "bf16", 4, 4, 2, 64, 64, False, (True, True))
    bad = [dict(q=dv["q"].float()), dict(k=dv["k"][:3]), dict(position=dv["position"].long()), dict(position=dv["position"][:3]),
           dict(q_weight=dv["q_weight"][:32]), dict(k_weight=dv["k_weight"].float()), dict(table=dv["table"].double()),
           dict(table=dv["table"][:, :, 0]), dict(q=dv["q"].cpu()), dict(position=None),
           dict(q=dv["q"].transpose(1, 2)), dict(table=torch.zeros(9, 40, 2, device=gpu_device)),
           dict(q=torch.zeros(4, 4, 65, dtype=torch.bfloat16, device=gpu_device)[..., 1:])]
    for change in bad:
        with pytest.raises(api.AtGrpoError):
            forward({**dv, **change}, False)
        with pytest.raises(api.AtGrpoError):
            backward({**dv, **change}, False)
    with pytest.raises(api.AtGrpoError):
        backward({**dv, "dq": dv["dq"][:, :2]}, False)
    for D in (12, 264):
        x = torch.zeros(4, 2, D, dtype=torch.bfloat16, device=gpu_device)
        with pytest.raises(api.AtGrpoError):
            api.at_grpo_qk_norm_rope(x, None, None, dv["position"])


def test_refusals_of_the_library_on_the_host():
    """Argument errors come back as a status, with nothing launched: no GPU is needed to see them."""
    lib, C = api.load_library(), api.C
    rows = api._Rows(4096, 64, 64)
    odd = [api._Rows(4100, 64, 64), api._Rows(4096, 65, 64), api._Rows(4096, 64, 4), api._Rows(0, 64, 64)]

    def layer(**kw):
        a = dict(dtype=1, D=64, rot_dim=64, layout=0, n_pos=10, eps=1e-6, table=4096, q_weight=4096, k_weight=4096)
        a.update(kw)
        return api._NormRope(*a.values())

    def call(L, n=4, hq=2, hk=2, q=rows, o=rows, pos=4096):
        return lib.at_grpo_qk_norm_rope(C.byref(L), n, hq, hk, C.byref(q), C.byref(rows), pos, C.byref(o), C.byref(rows), None, None)

    for kw, status in [(dict(dtype=2), 2), (dict(D=60), 2), (dict(D=0), 1), (dict(D=264), 2), (dict(rot_dim=66), 1), (dict(rot_dim=7), 1),
                       (dict(layout=2), 1), (dict(n_pos=0), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(table=None), 1),
                       (dict(table=4100), 1), (dict(q_weight=4100), 1)]:
        assert call(layer(**kw)) == status, kw
    assert call(layer(), n=-1) == 1 and call(layer(), hq=0, hk=0) == 1 and call(layer(), hq=-1) == 1 and call(layer(), pos=None) == 1
    assert call(layer(), n=0) == 0
    for r in odd:
        assert call(layer(), q=r) == 1 and call(layer(), o=r) == 1
    assert lib.at_grpo_qk_norm_rope(None, 0, 1, 1, None, None, None, None, None, None, None) == 1
    ws = lib.at_grpo_workspace_bytes(api.CALL_QK_NORM_ROPE_BWD, None, 0, 0, 0, 0)
    assert ws > 0
    r = C.byref(rows)

    def back(dqw=4096, w=4096, nbytes=ws, x=r):
        return lib.at_grpo_qk_norm_rope_bwd(C.byref(layer()), 4, 2, 2, r, r, x, r, 4096, r, r, dqw, 4096, None, w, nbytes, None)

    assert back(dqw=None) == 1 and back(x=None) == 1 and back(w=None) == 3 and back(w=4097) == 3 and back(nbytes=ws - 1) == 3
    for kw, status in [(dict(rot_dim=0), 1), (dict(rot_dim=3), 1), (dict(rot_dim=300), 2), (dict(base=0.0), 1), (dict(scaling=4), 1),
                       (dict(scaling=1, factor=0.5), 1), (dict(scaling=2, factor=2.0, rot_dim=2), 1), (dict(scaling=3, factor=2.0, trained=0.0), 1),
                       (dict(scaling=3, factor=2.0, trained=9.0, slow=2.0, fast=2.0), 1), (dict(magnitude=0.0), 1)]:
        a = dict(rot_dim=64, scaling=0, base=1e4, factor=1.0, trained=0.0, slow=1.0, fast=32.0, magnitude=1.0)
        a.update(kw)
        assert lib.at_grpo_rope_table(C.byref(api._Rope(*a.values())), 4, 4096, None) == status, kw
    assert lib.at_grpo_rope_table(None, 4, 4096, None) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,rot,inter", [(64, 0, False), (64, 32, False), (64, 32, True), (80, 20, False), (80, 50, True), (256, 192, False), (128, 2, False)])
@pytest.mark.parametrize("normed", [False, True])
def test_elements_that_do_not_turn(gpu_device, dtype, D, rot, inter, normed):
    """Behind rot_dim an element is its own: infinities, NaN and signs of zeros of one do not reach another, forward and in the gradient
    (with a norm, what goes into the row's size and mean reaches all of the row by the formula)."""
    c, dv = case(gpu_device, dtype, 7, 3, 2, D, rot, inter, (normed, normed), seed=3)
    dt = DTYPES[dtype]
    for name in ("q", "dq", "k", "dk"):
        x = c[name]
        if name.startswith("d") or not normed:
            x[0, 0, rot + 1], x[1, 1, D - 2], x[2, 0, rot], x[2, 0, D - 1] = np.inf, np.nan, -np.inf, np.inf
        x[3, 1, rot], x[3, 1, rot + 1] = -0.0, -1.5
        x[4, 0, rot], x[4, 0, rot + 1] = -0.0, 1.5
        dv[name] = to_dev(x, dt, gpu_device)
    out, grad = forward(dv, inter), backward(dv, inter)
    for name in ("q", "k"):
        args = c[name + "_weight"], c["table"], c["position"]
        with np.errstate(invalid="ignore"):
            ref = oracle.norm_rope(c[name], *args, 1e-5, inter)
            dx, dw = oracle.norm_rope_grad(c["d" + name], c[name], *args, 1e-5, inter)
        got, gx = host64(out[name]), host64(grad["d" + name])
        for mine, want in ((got, ref), (gx, dx)):
            assert np.array_equal(np.isnan(mine), np.isnan(want)) and np.array_equal(np.isinf(mine), np.isinf(want))
            assert np.array_equal(mine[np.isinf(mine)], want[np.isinf(want)])
            zero = want == 0
            assert np.array_equal(np.signbit(mine[zero]), np.signbit(want[zero]))
        if normed:
            assert np.array_equal(np.isnan(host64(grad[f"d{name}_weight"])), np.isnan(dw)) and np.array_equal(np.isinf(host64(grad[f"d{name}_weight"])), np.isinf(dw))
        else:
            keep = slice(rot, None)
            assert np.array_equal(got[..., keep], c[name][..., keep], equal_nan=True) and np.array_equal(gx[..., keep], c["d" + name][..., keep], equal_nan=True)


def test_more_heads_than_are_counted_are_refused_on_the_host():
    lib, C = api.load_library(), api.C
    r = C.byref(api._Rows(4096, 64, 64))
    L = C.byref(api._NormRope(1, 64, 0, 0, 0, 1e-6, None, 4096, 4096))
    ws = lib.at_grpo_workspace_bytes(api.CALL_QK_NORM_ROPE_BWD, None, 0, 0, 0, 0)
    kv = C.byref(api._KV(dtype=1, Hk=2, D=64, page_size=16, n_pages=9, n_seq=4, max_pages=3, n_group=0, max_prefix_pages=0, k=4096, v=4096, pages=4096, length=4096))
    most = (1 << 31) - 1
    for hq, hk in [(most, 0), (0, most), (most, most), (1 << 30, 1), (most - 100, 100)]:
        assert lib.at_grpo_qk_norm_rope(L, 4, hq, hk, r, r, None, r, r, None, None) == 2
        assert lib.at_grpo_qk_norm_rope_bwd(L, 4, hq, hk, r, r, r, r, None, r, r, 4096, 4096, None, 4096, ws, None) == 2
    for hq in (most, most - 4, 1 << 30):
        assert lib.at_grpo_kv_append(kv, L, 4, hq, r, r, r, r, None, None) == 2
    assert lib.at_grpo_qk_norm_rope(L, 4, -1, 2, r, r, None, r, r, None, None) == 1
    assert lib.at_grpo_qk_norm_rope_bwd(L, 4, 2, -1, r, r, r, r, None, r, r, 4096, 4096, None, 4096, ws, None) == 1


@pytest.mark.gpu
def test_more_rows_than_a_launch_counts_threads(gpu_device):
    """A wavefront a row: 7 * 10^7 rows are more than 2^32 threads."""
    n = 70_000_001
    x, w = torch.ones(n, 1, 8, dtype=torch.bfloat16, device=gpu_device), torch.full((8,), 2.0, dtype=torch.bfloat16, device=gpu_device)
    x[-1] = -1
    y = api.at_grpo_qk_norm_rope(x, None, None, None, w)["q"]      # 1 / sqrt(1 + 1e-6) rounds to 1
    assert (y[:-1] == 2).all() and (y[-1] == -2).all()
    out = api.at_grpo_qk_norm_rope_bwd(x, None, x, None, None, None, None)
    assert torch.equal(out["dq"], x)


@pytest.mark.parametrize("n_pos,rot_dim", [(1 << 31, 2), ((1 << 32) + 5, 2), (-1, 64), (4, 0), (4, -2), (4, 63), (0, (1 << 32) + 64), (4, 258)])
def test_tables_of_sizes_that_there_are_not(n_pos, rot_dim):
    """Before anything is allocated, and not modulo 2^32."""
    with pytest.raises(api.AtGrpoError):
        api.at_grpo_rope_table(n_pos, rot_dim)


def test_outputs_that_meet_their_inputs_otherwise_are_refused_on_the_host():
    lib, C = api.load_library(), api.C
    at, r = 1 << 24, lambda *a: C.byref(api._Rows(*a))
    L = C.byref(api._NormRope(1, 64, 0, 0, 0, 1e-6, None, 4096, 4096))
    ws = lib.at_grpo_workspace_bytes(api.CALL_QK_NORM_ROPE_BWD, None, 0, 0, 0, 0)
    kv = C.byref(api._KV(dtype=1, Hk=2, D=64, page_size=16, n_pages=9, n_seq=4, max_pages=3, n_group=0, max_prefix_pages=0, k=4096, v=4096, pages=4096, length=4096))
    there, far = r(at, 512, 64), r(at + (1 << 20), 512, 64)
    for other in (r(at + 64 * 2, 512, 64), r(at - 16, 512, 64), r(at + 512 * 2, 512, 64), r(at, 64, 512), r(at, 256, 64)):
        for a, b in ((there, other), (other, there)):
            assert lib.at_grpo_qk_norm_rope(L, 4, 4, 0, a, None, None, b, None, None, None) == 1
            assert lib.at_grpo_qk_norm_rope(L, 4, 0, 4, None, a, None, None, b, None, None) == 1
            assert lib.at_grpo_kv_append(kv, L, 4, 4, a, far, far, b, None, None) == 1
            assert lib.at_grpo_qk_norm_rope_bwd(L, 4, 4, 0, a, None, far, None, None, b, None, 4096, 4096, None, 4096, ws, None) == 1
            assert lib.at_grpo_qk_norm_rope_bwd(L, 4, 4, 0, far, None, a, None, None, b, None, 4096, 4096, None, 4096, ws, None) == 1
            assert lib.at_grpo_qk_norm_rope_bwd(L, 4, 0, 4, None, far, None, a, None, None, b, 4096, 4096, None, 4096, ws, None) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outputs_beside_and_over_their_inputs(gpu_device, dtype):
    c, dv = case(gpu_device, dtype, 21, 4, 2, 64, 64, False, (True, True))
    ref, gref = forward(dv, False), backward(dv, False)
    buffer = torch.zeros(24, 12, 64, dtype=DTYPES[dtype], device=gpu_device)
    rows = buffer[:21, 1:5]
    rows.copy_(dv["q"])
    for out in (buffer[:21, 4:8], buffer[:21, :4], buffer[3:, 1:5]):
        with pytest.raises(api.AtGrpoError):
            forward({**dv, "q": rows}, False, q_out=out)
        with pytest.raises(api.AtGrpoError):
            backward({**dv, "dq": rows}, False, dq=out)
    assert torch.equal(rows, dv["q"])
    forward({**dv, "q": rows}, False, q_out=buffer[:21, 5:9])      # between each other's rows
    assert torch.equal(buffer[:21, 5:9], ref["q"]) and torch.equal(rows, dv["q"])
    g = backward({**dv, "q": rows}, False, dq=rows)      # in place of the queries
    assert torch.equal(rows, gref["dq"]) and torch.equal(g["dq_weight"], gref["dq_weight"])
    assert not buffer[21:].any() and not buffer[:, 9:].any() and not buffer[:, 0].any()
