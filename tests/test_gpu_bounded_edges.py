"""The decayed and the windowed attention where their numbers leave the ordinary."""
import math

import pytest
import torch

from paper_2406_07368_amd import binding
from plain_attention import decay_prefill, near, window_attend, window_seen

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
NORM = {BF: None, F32: 5e-6}                     # as in test_gpu_decay.py


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


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("where", ["query", "infinite score", "key"])
def test_prompt_hands_on_what_is_not_finite(dtype, where):
    B, H, Hkv, L, d, W, sinks = 2, 4, 2, 300, 128, 100, 3
    q, = rows(B, H, L, d, dtype, 55)
    k, v = rows(B, Hkv, L, d, dtype, 65, 2)
    hit, t = torch.zeros((B, H, L), dtype=torch.bool), 150
    if where == "query":
        q[0, 1, t, 3] = math.nan
        hit[0, 1, t] = True
    elif where == "infinite score":
        q[0, 0, t + 20], k[0, 0, t] = 1e30, 1e30
        hit[0, 0, t + 20] = True
    else:
        k[0, 0, t, 5] = math.nan
        hit[0, :H // Hkv, t:t + W] = True
    out, lse, _ = binding.window_prefill(*cuda(q, k, v), W, sinks, 0.2, want_lse=True)
    assert bool(torch.isnan(out.cpu()[hit]).all()) and bool(torch.isnan(lse.cpu()[hit]).all())
    if where == "query":
        assert bool(torch.isfinite(out.cpu()[~hit]).all())
    assert bool(torch.isfinite(out[1]).all()) and bool(torch.isfinite(out[:, H // Hkv:]).all())


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


def calls_for_a_stream():
    """Calls that need a workspace, and calls that need none, of every kind; what each is given; as functions of the stream."""
    B, H, d, L, W = 1, 4, 64, 900, 1200
    q, k, v, do = cuda(*rows(B, H, L, d, BF, 71, 4))
    tok = cuda(*rows(B, H, 3, d, BF, 72, 3))
    held = cuda(*rows(B, H, W + 2, d, BF, 73, 2))
    g, w = torch.linspace(-1, -0.01, H, device="cuda"), torch.rand(H, d, 3, device="cuda")
    S, z, h = torch.randn(B, H, d, d, device="cuda"), torch.rand(B, H, d, device="cuda") + 9, cuda(*rows(B, H, 2, d, BF, 74))[0]
    parent = torch.tensor([-1, 0, 0], dtype=torch.int32, device="cuda")
    pos = torch.full((B, H), 3000, dtype=torch.int32, device="cuda")
    out, lse, _ = binding.window_prefill(q, k, v, W, 2, want_lse=True)
    x = dict(q=q, k=k, v=v, do=do, tq=tok[0], tk=tok[1], tv=tok[2], kc=held[0], vc=held[1], g=g, w=w, S=S, z=z, h=h, parent=parent, pos=pos, out=out, lse=lse)
    x.update({n + "512": x[n][:, :, :512].contiguous() for n in ("q", "k", "v", "do")} | {n + "1": x["t" + n][:, :, 0].contiguous() for n in "qkv"})

    def flat(r):
        return [y for x in r if x is not None for y in (flat(x) if isinstance(x, tuple) else [x])] if isinstance(r, tuple) else [r]

    return x, [lambda x, s, f=f: flat(f(x, s)) for f in (
        lambda x, s: binding.decay_prefill(x["q"], x["k"], x["v"], x["g"], state=x["S"], stream=s),
        lambda x, s: binding.decay_backward(x["q"], x["k"], x["v"], x["g"], x["do"], stream=s),
        lambda x, s: (binding.decay_step(x["tq"], x["tk"], x["tv"], x["g"], x["S"], stream=s), x["S"]),
        lambda x, s: binding.window_prefill(x["q"], x["k"], x["v"], W, 2, want_lse=True, stream=s),
        lambda x, s: (lambda r: (r[0], r[2][0][:, :, :L], r[2][1][:, :, :L], r[2][2]))(binding.window_prefill(x["q"], x["k"], x["v"], W, 2, want_cache=True, stream=s)),
        lambda x, s: binding.window_backward(x["q"], x["k"], x["v"], x["out"], x["lse"], x["do"], W, 2, stream=s),
        lambda x, s: (binding.window_step(x["tq"], x["tk"], x["tv"], (x["kc"], x["vc"], x["pos"]), W, 2, stream=s), x["kc"], x["vc"], x["pos"]),
        lambda x, s: binding.prefill(x["q"], x["k"], x["v"], x["w"], stream=s),
        lambda x, s: binding.prefill_grouped_backward(x["q512"], x["k512"], x["v512"], x["w"], x["do512"], group=64, stream=s),
        lambda x, s: (binding.verify(x["tq"], x["tk"], x["tv"], x["w"], (x["S"], x["z"], x["h"]), stream=s), x["S"], x["z"], x["h"]),
        lambda x, s: binding.verify_tree(x["tq"], x["tk"], x["tv"], x["parent"], x["w"], (x["S"], x["z"], x["h"]), stream=s),
        lambda x, s: binding.decode(x["q1"], x["k1"], x["v1"], x["w"], (x["S"], x["z"], x["h"]), stream=s))]


def test_memory_of_calls_on_a_stream():
    """Calls that wait on a busy stream, by its handle and as torch's: what they were given, their workspace and what they return is not
    handed out to the stream that goes on, which fills whatever memory it gets."""
    x, calls = calls_for_a_stream()
    copies = lambda: {n: t.clone() for n, t in x.items()}  # noqa: E731
    want = [[y.clone() for y in f(copies(), None)] for f in calls]
    side = torch.cuda.Stream()
    for handle in (side.cuda_stream, side):
        for i, f in enumerate(calls):
            given = copies()
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                keep_busy()
            got = f(given, handle)
            sizes = [t.numel() * t.element_size() for t in given.values()]
            del given
            spoilt = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes + [1 << e for e in range(9, 24)] for _ in range(2)]
            torch.cuda.synchronize()
            assert len(got) == len(want[i]) and all(torch.equal(a, b) for a, b in zip(got, want[i])), i
            del spoilt, got


def test_calls_on_a_stream_in_a_graph():
    """The capturing stream named in the call: the replays give the eager bits, with other work between."""
    x, calls = calls_for_a_stream()
    calls = [calls[i] for i in (0, 1, 3, 4, 5, 7, 8)]                   # (those that change nothing that they are given)
    want = [[y.clone() for y in f(x, None)] for f in calls]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = [f(x, side) for f in calls] + [f(x, side.cuda_stream) for f in calls]
    for i in range(4):
        for y in (z for h in held for z in h):
            y.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        for i, (h, w) in enumerate(zip(held, want + want)):
            assert all(torch.equal(a, b) for a, b in zip(h, w)), i
        [f(x, None) for f in calls]


def test_memory_that_the_current_stream_still_uses():
    """A call on an idle stream, while the current stream is behind and will still write to memory that was let go."""
    x, calls = calls_for_a_stream()
    copies = lambda: {n: t.clone() for n, t in x.items()}  # noqa: E731
    want = [[y.clone() for y in f(copies(), None)] for f in calls]
    side = torch.cuda.Stream()
    for handle in (side.cuda_stream, side, 0):
        for i, f in enumerate(calls):
            given = copies()
            torch.cuda.synchronize()
            if handle != 0:
                keep_busy()
            for n in [t.numel() * t.element_size() for w in want for t in w] + [1 << e for e in range(9, 24)]:
                torch.full((n,), 255, dtype=torch.uint8, device="cuda")
            got = f(given, handle)
            torch.cuda.synchronize()
            assert len(got) == len(want[i]) and all(torch.equal(a, b) for a, b in zip(got, want[i])), i


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kk,keep", [(1, 1), (4, 3)])
def test_thousands_of_steps(dtype, kk, keep):
    """Decays that no 32-bit factor near 1 meets exactly, on rows whose state only grows, against the recurrence in 64 bits."""
    g = torch.tensor([-1.3 * 2 ** -11, -1.3 * 2 ** -10, -1e-3, -1.7e-5, -0.03, -2.0, 0.0])
    B, H, d, n = 1, len(g), 64, 4096
    k, v = (torch.rand((n, B, H, kk, d), generator=torch.Generator().manual_seed(54 + i)).to(dtype).cuda() for i in range(2))
    gg, commit = g.cuda(), torch.full((B,), keep, dtype=torch.int32, device="cuda")
    S = torch.zeros((B, H, d, d), device="cuda")
    for t in range(n):
        binding.decay_step(k[t], k[t], v[t], gg, S, 1.0, commit)
    lam = torch.exp(g.double()).cuda()[:, None, None]
    want = torch.zeros((B, H, d, d), dtype=torch.float64, device="cuda")
    for t in range(n):
        for i in range(keep):
            want = lam * want + k[t, :, :, i, :, None].double() * v[t, :, :, i, None, :].double()
    for h in range(H):
        # A step rounds the sum of a state and what it gains, by at most 2^-24 of it and 2^-24 / sqrt(3) in the mean square,
        # independently of the others'; it weighs lambda^keep to the power of the steps that follow.  Twice that, for the
        # gain's own roundings and chance, and 2^-22 for the factor (1 - lambda), which is off by some 2^-23 of itself.
        lam2 = math.exp(2 * keep * float(g[h]))
        steps = n if lam2 == 1 else min(n, 1 / (1 - lam2))
        rel = float((S[0, h].double() - want[0, h]).norm() / want[0, h].norm())
        assert rel <= 2 * 2.0 ** -24 / math.sqrt(3) * math.sqrt(steps) + 2.0 ** -22, (float(g[h]), rel)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("L", [160, 1000])
def test_outliers_in_heads_that_forget_fast(dtype, L):
    """The last token of a group is 1e6 (bf16: 1e8) times the others, of 160 tokens the square of that: what is left of it after the
    next group is still right."""
    g = torch.tensor([-0.05, -0.1, -0.16, -0.2, -0.25, -0.3, -0.4, -0.5, -0.6])
    H, d = len(g), 64
    q, k, v = rows(1, H, L, d, dtype, 56, 3)
    for at in (63, L - 97):
        v[:, :, at] *= 1e8 if dtype == BF else 1e6
    want, S, size, A = decay_prefill(q.double(), k.double(), v.double(), g, 1.0)
    out, Sg = binding.decay_prefill(*cuda(q, k, v, g), 1.0)
    near(out, want, size, dtype, 2 if dtype == BF else 200, "out", NORM[dtype])
    off = (Sg.double().cpu() - S).abs() - 2.0 ** -18 * A
    assert float(off.max()) <= 0


@pytest.mark.parametrize("H,Hkv,d,W,sinks", [(4, 2, 64, 30, 2), (4, 1, 128, 500, 0), (2, 2, 128, 1, 1)])
def test_gradient_of_a_sequence_of_one_token_in_a_batch(H, Hkv, d, W, sinks):
    """Its softmax is over one key and constant: dq and dk are 0, as they are where the token comes alone."""
    B, L = 3, 300
    q, do = cuda(*rows(B, H, L, d, BF, 57, 2))
    k, v = cuda(*rows(B, Hkv, L, d, BF, 58, 2))
    lens = torch.tensor([1, L, 1], dtype=torch.int32, device="cuda")
    out, lse, _ = binding.window_prefill(q, k, v, W, sinks, 3.0, lens, want_lse=True)
    dq, dk, dv = binding.window_backward(q, k, v, out, lse, do, W, sinks, 3.0, lens)
    for b in (0, 2):
        one = [x[b:b + 1, :, :1].contiguous() for x in (q, k, v, out, do)]
        gq, gk, gv = binding.window_backward(*one[:4], lse[b:b + 1, :, :1].contiguous(), one[4], W, sinks, 3.0)
        assert not dq[b].any() and not dk[b].any() and not gq.any() and not gk.any()
        assert torch.allclose(dv[b, :, :1].float(), gv[0].float(), rtol=2.0 ** -7, atol=0)     # (shares added up in another order: one step of bf16)


@pytest.mark.parametrize("B,H,Hkv,L,d,W,sinks,ragged", [
    (2, 2, 1, 1, 128, 5, 3, False), (1, 2, 2, 31, 128, 7, 0, False), (2, 4, 2, 65, 128, 1, 0, True), (1, 2, 1, 129, 64, 1, 64, False),
    (2, 2, 1, 300, 64, 5, 2, True), (1, 4, 2, 200, 128, 2, 0, False), (2, 24, 3, 85, 128, 8, 1, True)])
def test_gradient_of_narrow_windows_in_the_norm(B, H, Hkv, L, d, W, sinks, ragged):
    """dq and dk of windows of 8 tokens and fewer, exactly 0 where every token sees only itself."""
    q, do = rows(B, H, L, d, BF, 59, 2)
    k, v = rows(B, Hkv, L, d, BF, 60, 2)
    lens = torch.tensor([L, L // 2 + 1][:B], dtype=torch.int32) if ragged else None
    live = torch.ones((B, 1, L, 1), dtype=torch.bool) if lens is None else (torch.arange(L) < lens[:, None])[:, None, :, None]
    x = [t.double().requires_grad_() for t in (q, k, v)]
    G = H // Hkv
    Q, K, V = (torch.where(live, t, 0.0) for t in x)
    t = torch.arange(L)
    out = window_attend(Q, K, V, window_seen(t[None], t[:, None], W, sinks), 0.2)[0]
    want = torch.autograd.grad(torch.where(live, out, 0.0), x, do.double())
    a = cuda(q, k, v, do, lens)
    o, lse, _ = binding.window_prefill(*a[:3], W, sinks, 0.2, a[4], want_lse=True)
    for n, g, w in zip("qkv", binding.window_backward(*a[:3], o, lse, a[3], W, sinks, 0.2, a[4]), want):
        if n != "v" and (L == 1 or W == 1 and sinks == 0):
            assert not g.any()
            continue
        # two independent roundings to bf16, dS (or P) and the result, each 2^-8 / sqrt(3) at most in the mean square
        assert float((g.double().cpu() - w).norm()) <= math.sqrt(2 / 3) * 2.0 ** -8 * float(w.norm()), n


@pytest.mark.parametrize("B,H,Hkv,d,kk,W,sinks,pos", STEPS)
def test_steps_of_bf16_rows_are_off_by_their_own_rounding(B, H, Hkv, d, kk, W, sinks, pos):
    q, k, v, kc, vc, P = step_case(BF, B, H, Hkv, d, kk, W, sinks, pos)
    a = cuda(q, k, v, kc, vc, P)
    got = binding.window_step(*a[:3], tuple(a[3:]), W, sinks, 0.2).double().cpu()
    held = torch.tensor([s if s < sinks else sinks + (s - sinks) % W for s in range(pos) if s < sinks or s >= pos - W])
    at = torch.tensor([s for s in range(pos) if s < sinks or s >= pos - W])
    K, V = (torch.cat([x[:, :, held], y], 2).double() for x, y in ((kc, k), (vc, v)))
    new = pos + torch.arange(kk)
    want, _, size = window_attend(q.double(), K, V, window_seen(torch.cat([at, new])[None], new[:, None], W, sinks), 0.2)
    # a weight is off by 2^-8 of its second term, which is 2^-8 of it at most; fp32 sums as in plain_attention.near
    assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -16 + 2.0 ** -18) * size).all())
    assert float((got - want).norm()) <= float((want.to(BF).double() - want).norm()) + 2.0 ** -16 * float(size.norm())
