"""Log-sums and best tokens where the largest logit over the temperature is far from the range of exponents, and beside NaN of either kind."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as oracle
from paper_2510_11062_amd import api
from tests.rollout_case import DTYPES, U32, rounded, to_dev
from tests.test_gpu_logit_rules import Rows, apply, compare, draw

TEMPERATURES = [1e-3, 1e-5, 1e-6, 1e-7, 1e-8, 1e-9, 1e-10, 1e-12, 1e-20, 1e-30]
LEVELS = [1e6, 1e7, 1e8, 1e9, 1e10, 3e12, 1e20, 1e29]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [33, 2048, 8195, 20001])
def test_small_temperatures(gpu_device, dtype, V):
    rs = np.random.default_rng(V)
    n = 3 * len(TEMPERATURES)
    r = Rows(rounded(rs.normal(size=(n, V)) * 2.5, DTYPES[dtype]), DTYPES[dtype], temperature=np.repeat(TEMPERATURES, 3))
    r.logits[::3] += 20      # far from 0, and below it
    r.logits[1::3] -= 20
    r.logits = rounded(r.logits, r.dtype)
    word = torch.zeros(1, dtype=torch.int32, device=gpu_device)
    compare(apply(r, gpu_device, data_error=word, out_dtype=torch.float32), r.want(), what="temperature alone")
    assert int(word) == 0
    all_rules = draw(rs, dtype, V, n, [1 + i % 2 for i in range(n)], (n // 2, n - n // 2))
    all_rules.temperature = r.temperature
    compare(apply(all_rules, gpu_device, data_error=word), all_rules.want(), what="all rules")
    assert int(word) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [33, 2048, 8195, 20001])
def test_large_logits(gpu_device, dtype, V):
    """Of either sign, close to each other; the largest is no power of two."""
    rs = np.random.default_rng(V + 1)
    n = 2 * len(LEVELS)
    level = np.repeat(LEVELS, 2) * np.tile([1, -1], len(LEVELS))
    r = Rows(rounded(level[:, None] * (1.3 + 0.01 * rs.normal(size=(n, V))), DTYPES[dtype]), DTYPES[dtype])
    compare(apply(r, gpu_device), r.want(), what="no rule")
    r.temperature = rs.uniform(0.3, 2, n)
    compare(apply(r, gpu_device), r.want(), what="temperature")
    r.logits[:, V // 2] = 0      # and with one far from the others
    compare(apply(r, gpu_device), r.want(), what="one apart")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ban", [-1e7, -1e10, -1e20])
def test_rows_banned_whole(gpu_device, dtype, ban):
    V = 300
    rs = np.random.default_rng(5)
    r = Rows(rounded(rs.normal(size=(4, V)) * 2.5, DTYPES[dtype]), DTYPES[dtype], temperature=np.array([0.8, 1.0, 1.3, 0.01]))
    r.bias = [[(v, ban * (1 + 0.1 * s)) for v in range(V)] for s in range(4)]
    compare(apply(r, gpu_device, out_dtype=torch.float32), r.want())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(2100, 8192), (1400, 20001), (700, 50003)])
def test_small_temperatures_in_many_rows(gpu_device, dtype, n, V):
    """Workgroups with a chunk or several, rows of one workgroup and of several.  Bounds as `compare` has them, of temperature alone."""
    gen = torch.Generator(device=gpu_device).manual_seed(V)
    logits = (torch.randn(n, V, generator=gen, device=gpu_device) * 2.5).to(DTYPES[dtype])
    temperature = torch.tensor(TEMPERATURES, device=gpu_device).repeat(n // len(TEMPERATURES))
    assert len(temperature) == n
    o = api.at_grpo_logit_rules(api.LogitRules(temperature=temperature), logits, want_out=False)
    assert bool(torch.isfinite(o["lse"]).all())
    for rows in torch.arange(n, device=gpu_device).split(200):
        x = logits[rows].double() / temperature[rows].double()[:, None]
        lse, most = torch.logsumexp(x, 1), x.abs().amax(1)
        bound = U32 * (2.02 * most + 8 * most + 50 + V / 8192 + 8 * lse.abs())
        off = (o["lse"][rows].double() - lse).abs()
        assert bool((off <= bound).all()), f"{float((off / bound).max())} times the bound"


# ---- NaN ------------------------------------------------------------------------------------------------
# bits of a NaN that signals (the first bit of its mantissa is 0), and of one that does not
SIGNALLING = {"bf16": [0x7f81, 0x7fa0, -0x007f], "f32": [0x7f800001, 0x7fa00000, -0x007fffff]}
QUIET = {"bf16": [0x7fc0, -0x0040], "f32": [0x7fc00000, -0x00400000]}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["signalling", "quiet"])
@pytest.mark.parametrize("V", [40, 2048, 8200])
def test_the_best_beside_nan(gpu_device, dtype, kind, V):
    """A NaN is passed over by best, wherever among eight neighbours it and the largest stand, and whatever rules there are; lse is NaN, or where a
    mask takes the NaN out what is left has it."""
    ints = torch.int16 if dtype == "bf16" else torch.int32
    rs = np.random.default_rng(V)
    for bits in (SIGNALLING if kind == "signalling" else QUIET)[dtype]:
        for first in (0, V // 16 * 8, V - 8):
            at = [(first + i, first + j) for i in range(8) for j in range(8) if i != j]
            logits = to_dev(rounded(rs.normal(size=(len(at), V)), DTYPES[dtype]), DTYPES[dtype], gpu_device)
            rows = torch.arange(len(at), device=gpu_device)
            nan, best = (torch.tensor(x, device=gpu_device) for x in zip(*at))
            logits[rows, best] = 100.0
            plain = logits.clone()
            logits.view(ints)[rows, nan] = bits
            assert bool(torch.isnan(logits[rows, nan]).all()) and bool((logits.view(ints)[rows, nan] == bits).all())
            n = len(at)
            zeros = torch.zeros(n, 1, dtype=torch.int32, device=gpu_device)
            one = torch.ones(n, dtype=torch.int32, device=gpu_device)
            lists = dict(tokens=zeros + (first + 9) % V, length=one, presence=torch.full((n,), 0.5, device=gpu_device))
            biases = dict(bias_cu=torch.arange(n + 1, dtype=torch.int32, device=gpu_device), bias_token=one * ((first + 11) % V),
                          bias=torch.full((n,), -0.5, device=gpu_device))
            for rules in (api.LogitRules(), api.LogitRules(**lists), api.LogitRules(**lists, **biases), api.LogitRules(**biases)):
                o = api.at_grpo_logit_rules(rules, logits)
                assert torch.equal(o["best"].long(), best), (first, bits)
                assert bool(torch.isnan(o["lse"]).all()) and bool(torch.isnan(o["out"][rows, nan]).all())
                assert int(torch.isnan(o["out"]).sum()) == n
            # masked
            words = torch.full((n, (V + 31) // 32), -1, dtype=torch.int32, device=gpu_device)
            words[rows, nan // 32] = (-1 ^ (1 << (nan % 32))).to(torch.int32)
            rules = api.LogitRules(allowed=words, mask_row=rows.to(torch.int32))
            got, want = api.at_grpo_logit_rules(rules, logits), api.at_grpo_logit_rules(rules, plain)
            assert all(torch.equal(got[name], want[name]) for name in ("out", "lse", "best")) and torch.equal(got["best"].long(), best)


def test_the_oracle_passes_nan_over():
    out, lse, best, _ = oracle.sampling_row(np.array([1.0, np.nan, 5.0]), [], [], 1, 0, 0, 1, {}, None)
    assert best == 2 and np.isnan(lse) and np.isnan(out[1])
    assert oracle.sampling_row(np.array([1.0, np.nan, 5.0]), [], [], 1, 0, 0, 1, {}, np.array([True, False, True]))[1] == pytest.approx(5 + np.log1p(np.exp(-4)))
