"""Log-sums where the largest logit over the temperature is far from the range of exponents."""
import numpy as np
import pytest
import torch

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
