"""The decayed and the windowed attention where their numbers leave the ordinary."""
import math

import pytest
import torch

from paper_2406_07368_amd import binding

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def rows(B, H, L, d, dtype, seed, n=1):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((B, H, L, d), generator=g).to(dtype) for _ in range(n)]


def cuda(*xs):
    return [None if x is None else x.cuda() for x in xs]


# workgroups that share a head's cache, and one that has it to itself (few rows; many heads)
STEPS = [(2, 8, 2, 128, 1, 500, 4, 900), (2, 4, 2, 64, 5, 700, 0, 650), (1, 8, 8, 64, 16, 300, 64, 2000), (2, 8, 2, 128, 2, 20, 3, 100), (260, 4, 4, 64, 1, 80, 1, 90)]


def step_case(dtype, B, H, Hkv, d, kk, W, sinks, pos):
    q, = rows(B, H, kk, d, dtype, 51)
    k, v = rows(B, Hkv, kk, d, dtype, 52, 2)
    kc, vc = rows(B, Hkv, sinks + W, d, dtype, 53, 2)
    return q, k, v, kc, vc, torch.full((B, Hkv), pos, dtype=torch.int32)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,H,Hkv,d,kk,W,sinks,pos", STEPS)
@pytest.mark.parametrize("where", ["query", "infinite score", "key", "value", "value of no weight"])
def test_step_hands_on_what_is_not_finite(dtype, B, H, Hkv, d, kk, W, sinks, pos, where):
    """A NaN or a score of +inf makes NaN of the output rows that see it, however many workgroups share the cache."""
    q, k, v, kc, vc, P = step_case(dtype, B, H, Hkv, d, kk, W, sinks, pos)
    G = H // Hkv
    seen = sinks + (pos - 1 - sinks) % W                     # the newest token's ring row, which every draft sees (kk < window)
    hit = torch.zeros((B, H, kk), dtype=torch.bool)
    clean = cuda(q, k, v, kc, vc, P)
    want = binding.window_step(*clean[:3], tuple(clean[3:]), W, sinks, 0.2, torch.zeros(B, dtype=torch.int32, device="cuda"))
    if where == "query":
        q[0, 1, 0, 3] = math.nan
        hit[0, 1, 0] = True
    elif where == "infinite score":
        q[0, 0, kk - 1], kc[0, 0, seen] = 1e30, 1e30
        hit[0, 0, kk - 1] = True
    else:
        if where == "key":
            kc[0, 0, seen, 5] = math.nan
        elif where == "value":
            vc[0, 0, seen] = math.nan
        else:
            q[0, :G, :, 0], kc[0, 0, seen, 0], vc[0, 0, seen] = 100.0, -100.0, math.nan
        hit[0, :G] = True
    a = cuda(q, k, v, kc, vc, P)
    got = binding.window_step(*a[:3], tuple(a[3:]), W, sinks, 0.2, torch.zeros(B, dtype=torch.int32, device="cuda"))
    assert bool(torch.isnan(got.cpu()[hit]).all())
    others = [h for h in range(H) if h // G != (1 // G if where == "query" else 0)]
    assert torch.equal(got[1:], want[1:]) and torch.equal(got[:, others], want[:, others])
    if where == "query":
        assert bool(torch.isfinite(got.cpu()[~hit]).all())


def keep_busy():
    """Some 50 ms of work on the current stream."""
    x = torch.ones((8192, 8192), dtype=BF, device="cuda")
    for _ in range(60):
        x @ x


@pytest.mark.parametrize("L", [90, 0])
def test_cache_of_a_prompt_on_another_stream(L):
    """Nothing of the call runs on the current stream, which is behind: pos says how long the prompts are."""
    B, H, Hkv, d, W, sinks = 3, 4, 2, 64, 40, 2
    q, = cuda(*rows(B, H, L, d, BF, 61))
    k, v = cuda(*rows(B, Hkv, L, d, BF, 62, 2))
    tok = cuda(*rows(B, H, 1, d, BF, 63), *rows(B, Hkv, 1, d, BF, 64, 2))
    lens = torch.tensor([L, L // 3, 0], dtype=torch.int32, device="cuda")
    _, _, cache = binding.window_prefill(q, k, v, W, sinks, lens=lens, want_cache=True)
    assert cache[2].tolist() == [[n] * Hkv for n in lens.tolist()]
    want = binding.window_step(*tok, cache, W, sinks)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    keep_busy()
    _, _, cache = binding.window_prefill(q, k, v, W, sinks, lens=lens, want_cache=True, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert cache[2].tolist() == [[n] * Hkv for n in lens.tolist()]
    assert torch.equal(binding.window_step(*tok, cache, W, sinks), want)
