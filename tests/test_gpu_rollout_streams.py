"""The calls in front of the head on another stream than the one their tensors were made on, and in captured graphs: the bits of the eager
calls, in every replay, with eager work between the replays."""
import pytest
import torch

from paper_2510_11062_amd import api
from tests.rollout_case import DTYPES, Paged, to_dev


def bits(x):
    return {k: t.clone() for k, t in x.items() if isinstance(t, torch.Tensor) and k != "workspace"}


def same(a, b):
    return all(torch.equal(a[k], b[k]) for k in b)


def capture(fn, dev):
    side, g = torch.cuda.Stream(device=dev), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fn()      # the stream's workspace
    side.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            out = fn()
    return g, out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_and_rotation(gpu_device, dtype):
    gen = torch.Generator().manual_seed(0)
    rand = lambda *s: torch.randn(*s, generator=gen).to(DTYPES[dtype]).to(gpu_device)
    q, k, dq, dk, qw, kw = rand(500, 6, 64), rand(500, 2, 64), rand(500, 6, 64), rand(500, 2, 64), rand(64), rand(64)
    rope = api.at_grpo_rope_table(600, 64, device=gpu_device)
    position = torch.arange(500, dtype=torch.int32, device=gpu_device)
    forward = lambda: api.at_grpo_qk_norm_rope(q, k, rope, position, qw, kw)
    backward = lambda: api.at_grpo_qk_norm_rope_bwd(dq, dk, q, k, rope, position, qw, kw)
    for fn in (forward, backward):
        g, out = capture(fn, gpu_device)
        for step in range(3):
            position.copy_((torch.arange(500) * (step + 2)) % 600)
            q.mul_(1.25)
            want = bits(fn())
            for t in bits(out):
                out[t].fill_(7)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert same(out, want), step
        side = torch.cuda.Stream(device=gpu_device)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = fn()
        side.synchronize()
        assert same(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_decoded_token_as_a_graph(gpu_device, dtype):
    # lengths rise inside the graph, so that every replay is the next token: against the same tokens eagerly, in a cache of their own
    p = Paged(dtype, 2, 128, 16, [40, 100, 7, 64], None, [2, 2], [300, 90], seed=11, spare_columns=0)
    kv, other = p.device(gpu_device), p.device(gpu_device)
    start = kv.length - 6
    gen = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=gen).to(p.dtype).to(gpu_device)
    q, k, v, w = rand(4, 8, 128), rand(4, 2, 128), rand(4, 2, 128), rand(128)
    rope = api.at_grpo_rope_table(512, 128, device=gpu_device)

    def token(kv):
        kv.length += 1
        turned = api.at_grpo_kv_append(kv, q, k, v, rope, w, w)["q"]
        return api.at_grpo_prefix_attention(kv, turned, want_lse=True)

    kv.length.copy_(start)
    g, out = capture(lambda: token(kv), gpu_device)
    for batch in (kv, other):
        batch.length.copy_(start)
    for step in range(6):
        for x in (q, k, v):
            x.mul_(-1.125)
        want = bits(token(other))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert same(out, want), step
        assert torch.equal(kv.length, other.length)
    n = int(p.length[1])
    for a, b in ((kv.cache_k, other.cache_k), (kv.cache_v, other.cache_v)):
        page = int(p.pages[1][(n - 1) // 16])
        assert torch.equal(a[page, :, (n - 1) % 16], b[page, :, (n - 1) % 16])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("groups", [False, True])
def test_many_queries_as_a_graph(gpu_device, dtype, D, groups):
    p = Paged(dtype, 2, D, 16, [80, 200, 70, 64], [40, 70, 33, 64], *(([2, 2], [300, 90]) if groups else ()), seed=12)
    kv = p.device(gpu_device)
    q = to_dev(p.queries(4), p.dtype, gpu_device)
    fn = lambda: api.at_grpo_prefix_attention(kv, q, max_q=70, want_lse=True)
    g, out = capture(fn, gpu_device)
    for step in range(3):
        q.mul_(1.25)
        want = bits(fn())
        out["out"].fill_(9)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert same(out, want), step
